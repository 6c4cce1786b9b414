"""The matrix products of linear attention in the code that the compiler makes of it: behind a branch it has left out wait
states between a product and the first instruction that reads or overwrites the product's registers.  The source gives
them by hand there; this follows every way through the code from every product."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2608_21952_amd import build as libbuild

pytestmark = pytest.mark.skipif(shutil.which(libbuild.hipcc()) is None and
                                not os.path.exists(libbuild.hipcc()), reason="hipcc missing")

# What the compiler leaves within a block.
NEEDED = {"v_mfma_f32_16x16x32_f16": 8, "v_mfma_f32_16x16x32_bf16": 8, "v_mfma_f32_16x16x4_f32": 10}
FAR = 24   # wait states behind which nothing is looked for


def registers(text):
    out = set()
    for kind, first, last, one in re.findall(r"\b([va])(?:\[(\d+):(\d+)\]|(\d+)\b)", text):
        out |= {(kind, int(one))} if one else {(kind, i) for i in range(int(first), int(last) + 1)}
    return out


def kernels(assembly):
    """(name, instructions, places of the labels) of every kernel; an instruction is its name, operands and line."""
    name, code, labels = None, [], {}
    for number, line in enumerate(assembly.splitlines(), 1):
        line = line.split(";")[0].strip()
        label = re.match(r"(\S+):$", line)
        if label and label.group(1).startswith("_Z"):
            name, code, labels = label.group(1), [], {}
        elif label:
            labels[label.group(1)] = len(code)
        elif line.startswith(".end_amdhsa_kernel"):
            if code:
                yield name, code, labels
            code = []
        elif line and not line.startswith("."):
            op, _, rest = line.partition(" ")
            code.append((op, rest, number))


def first_uses(code, labels, start):
    """Wait states between the product at start and each first use of its result, over all ways, with the user's line."""
    result = registers(code[start][1].split(",")[0])
    ways, seen = [(start + 1, 0)], {}
    while ways:
        at, waited = ways.pop()
        while at < len(code) and waited < FAR and seen.get(at, FAR) > waited:
            seen[at] = waited
            op, rest, line = code[at]
            if op.startswith("v_mfma"):
                parts = rest.split(",")
                if registers(",".join(parts[1:3])) & result:
                    yield waited, line
                    break
                if registers(parts[0]) & result:   # sums on: the products wait for one another
                    break
            elif registers(rest) & result:
                yield waited, line
                break
            if op == "s_endpgm":
                break
            waited += int(rest, 0) + 1 if op == "s_nop" else 1
            if op == "s_branch":
                at = labels[rest.strip()]
                continue
            if op.startswith("s_cbranch"):
                ways.append((labels[rest.strip()], waited))
            at += 1


def too_early(assembly):
    found, products = [], 0
    for name, code, labels in kernels(assembly):
        for i, (op, _, line) in enumerate(code):
            if op.startswith("v_mfma"):
                products += 1
                found += [(name, op, line, use, waited) for waited, use in first_uses(code, labels, i) if waited < NEEDED[op]]
    return found, products


@pytest.fixture(scope="module")
def assembly():
    cmd = [libbuild.hipcc(), *libbuild.flags_for("linear_attention.hip"), "-S", "--cuda-device-only", "-o", "-",
           os.path.join(libbuild.CSRC, "linear_attention.hip")]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    return r.stdout


def test_no_use_is_too_early(assembly):
    found, products = too_early(assembly)
    assert products > 1000
    assert not found, f"{len(found)} of {products} products: {found[:3]}"


def test_stores_of_16_bytes_have_no_scalar_offset(assembly):
    """With one in a register the compiler leaves out the wait state in front of the next write to the data's registers."""
    stores = re.findall(r"buffer_store_dwordx4 [^\n;]*", assembly)
    assert stores
    for store in stores:
        assert store.split(",")[3].split()[0] == "0", store


def test_the_search_finds_one():
    """Over the branch the result is read three wait states behind its product, past it eight."""
    text = """_Z1k:
	v_mfma_f32_16x16x32_bf16 v[0:3], v[4:7], v[8:11], v[0:3]
	s_and_b64 vcc, exec, s[8:9]
	s_cbranch_vccnz .LBB0_2
	s_nop 4
.LBB0_2:
	s_add_u32 s0, s0, s1
	v_mul_f32_e32 v12, v1, v13
	s_endpgm
	.end_amdhsa_kernel
"""
    assert too_early(text) == ([("_Z1k", "v_mfma_f32_16x16x32_bf16", 2, 8, 3)], 1)
