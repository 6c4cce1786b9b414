// Rows into blocks of 32 values that share a power of two: e4m3 or e2m1 elements (mx.hpp), K filled up with zeros
// to whole blocks.  A block's values lie in four neighbouring lanes, eight in each.
// What bounds it: bytes, one read and one write; 16384 x 2560 fp16 to e2m1 26 us (4.1 TB/s).
#include "mx.hpp"

namespace ssdi8 {

namespace {

// A thread takes vectors kStep apart, kUnroll of them on their way at once.
constexpr int kUnroll = 4;

template <typename T, int kFormat>
__global__ __launch_bounds__(256) void quantize_mx_kernel(const T* x, int64_t x_row, int64_t rows, int k,
                                                          int row_vecs, uint8_t* codes, uint8_t* scales, int64_t from) {
  constexpr int kBytes = kFormat == SSDI8_FMT_MXFP8 ? kVec : kVec / 2;
  const int64_t total = rows * row_vecs;
  const int64_t first = (from + blockIdx.x) * (256 * kUnroll) + threadIdx.x;
  float v[kUnroll][kVec];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const int64_t i = first + u * 256;
    const int64_t row = i / row_vecs;
    const int o = (int)(i - row * row_vecs) * kVec;
    if (i < total) load_vec<T>(x + row * x_row + o, k - o, v[u]);
  }
  // whole quads have a vector: total is a multiple of 4
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const int64_t i = first + u * 256;
    if (i < total) mx_put<kFormat>(v[u], codes + i * kBytes, scales + i / 4, true);
  }
}

}  // namespace

hipError_t launch_quantize_mx(int dtype, int format, int64_t rows, int64_t k, const void* x, int64_t x_row,
                              void* codes, void* scales, hipStream_t st) {
  const int row_vecs = (int)(mx_blocks(k) * (kMxBlock / kVec));
  const int64_t workgroups = (rows * row_vecs + 256 * kUnroll - 1) / (256 * kUnroll);
  auto go = [&](auto t, auto f) {
    typedef decltype(t) T;
    return in_parts(workgroups, 256, [&](int64_t from, dim3 grid) {
      quantize_mx_kernel<T, decltype(f)::value>
          <<<grid, 256, 0, st>>>(static_cast<const T*>(x), x_row, rows, (int)k, row_vecs,
                                 static_cast<uint8_t*>(codes), static_cast<uint8_t*>(scales), from);
    });
  };
  auto by_type = [&](auto f) {
    switch (dtype) {
      case SSDI8_F32: return go(0.0f, f);
      case SSDI8_F16: return go((_Float16)0.0f, f);
      default: return go((bf16)0.0f, f);
    }
  };
  return format == SSDI8_FMT_MXFP8 ? by_type(std::integral_constant<int, SSDI8_FMT_MXFP8>())
                                   : by_type(std::integral_constant<int, SSDI8_FMT_MXFP4>());
}

}  // namespace ssdi8
