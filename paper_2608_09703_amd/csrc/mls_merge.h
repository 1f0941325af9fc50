// Merge of the forward's partial records into per-row statistics.
#pragma once

#include "mls_device.h"
#include "mls_launch.h"

namespace mls {

// Running merge of partial rows. Every sub-model keeps its own max m,
// sum exp(l - m) (s1) and sum exp((l - m) / tau) (st); the cross terms xr of
// every sub-model are weighted by the teacher's exponentials, so they are
// rescaled with the teacher's max. Slots follow the processing order, slot 0
// being the teacher; MM (the number of sub-models) is a compile-time constant,
// so every array is indexed with constants and stays in registers.
template <int MM>
struct RowState {
  float m[MM];
  float s1[MM];
  float st[MM];
  float xr[MM];
};

// rec[k] = partial of slot k over one vocabulary range (the same for all k)
template <int MM>
__device__ __forceinline__ void absorb(RowState<MM>& st, float ct, const float4* rec) {
  const float ms_new = fmaxf(st.m[0], rec[0].x);
  const float wa = fast_exp2((st.m[0] - ms_new) * ct);
  const float wb = fast_exp2((rec[0].x - ms_new) * ct);
#pragma unroll
  for (int k = 0; k < MM; ++k) {
    const float mo = st.m[k];
    const float mn = fmaxf(mo, rec[k].x);
    st.s1[k] = st.s1[k] * fast_exp2((mo - mn) * kLog2e) + rec[k].y * fast_exp2((rec[k].x - mn) * kLog2e);
    st.st[k] = st.st[k] * fast_exp2((mo - mn) * ct) + rec[k].z * fast_exp2((rec[k].x - mn) * ct);
    st.xr[k] = st.xr[k] * wa + rec[k].w * wb;
    st.m[k] = mn;
  }
}

// 4 tokens x 64 groups: 25 records per thread at the headline shape rather than
// 49 with 8 x 32 (row merge 39 -> 34 us per launch)
constexpr int kRowTok = 4;    // tokens per block
constexpr int kRowGrp = 64;   // partial groups per token, merged pairwise in a fixed tree
static_assert(kRowTok * kRowGrp == kThreads && (kRowGrp & (kRowGrp - 1)) == 0, "row merge shape");
static_assert(kFusedBN % kRowTok == 0, "a block's tokens lie in one token tile");

}  // namespace mls
