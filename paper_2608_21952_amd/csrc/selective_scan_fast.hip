// The selective scan's kernel (described in selective_scan.hip) with types and layouts fixed at compile time.
#include "selective_scan.hpp"

namespace ssdi8 {
namespace sel_scan {

namespace {

template <int kLanes, int kS, int kTile, int kSV, bool kTied> hipError_t by_type(Args& p, hipStream_t st) {
  const bool f32 = p.s.dt_dtype == 0;
  switch (p.s.dtype) {
    case 0: return launch_form<kLanes, kS, kTile, kSV, kTied, 0, 0, true>(p, st);
    case 1: return f32 ? launch_form<kLanes, kS, kTile, kSV, kTied, 1, 0, true>(p, st)
                       : launch_form<kLanes, kS, kTile, kSV, kTied, 1, 1, true>(p, st);
    default: return f32 ? launch_form<kLanes, kS, kTile, kSV, kTied, 2, 0, true>(p, st)
                        : launch_form<kLanes, kS, kTile, kSV, kTied, 2, 2, true>(p, st);
  }
}

}  // namespace

bool launch_fast(Args& p, hipStream_t st, hipError_t* e) {
  const SelScan& a = p.s;
  if (p.group_ch < kVec || a.dstate < kVec || a.dstate % 4 != 0) return false;
  if (a.tied) {
    if (a.headdim % kVec != 0 || p.group_ch % kVec != 0 || a.dstate <= 32 || a.dstate > 128) return false;
    *e = a.dstate <= 64 ? by_type<16, 4, 32, 2, true>(p, st) : by_type<16, 8, 32, 2, true>(p, st);
  } else {
    if (a.headdim != 1 || a.dstate > 32) return false;
    *e = a.dstate <= 16 ? by_type<8, 2, 64, 8, false>(p, st) : by_type<8, 4, 64, 8, false>(p, st);
  }
  return true;
}

}  // namespace sel_scan
}  // namespace ssdi8
