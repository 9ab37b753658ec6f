// The partial results of a shared-prefix decode and their join: per (sequence, head) `n_pre + splits` of them - the prefix's,
// then those of the sequence's own rows - each head_dim floats (a normalised output) and a log2-sum-exp, hd + 4 floats apart.
// Internal to the library.
#pragma once

#include "bt_common.cuh"
#include "bt_kernels.h"

namespace bt {
namespace parts {

// the lane's 8 dims of partials 0 .. count-1, `stride` of them apart
template <int HD, int WIDE>
__device__ __forceinline__ void fold_partials(SoftmaxState& st, const float* ws, int count, int stride, int sub)
{
    // WIDE at a time, all requested before the first is used
    for (int i0 = 0; i0 < count; i0 += WIDE) {
        float lse[WIDE];
        float4 x[WIDE], y[WIDE];
#pragma unroll
        for (int i = 0; i < WIDE; ++i) {
            const float* p = ws + (size_t)(i0 + i) * stride * (HD + 4);
            const bool there = i0 + i < count;
            lse[i] = there ? __ldcg(p + HD) : kNegInf;
            x[i] = y[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (there) {
                x[i] = __ldcg(reinterpret_cast<const float4*>(p + sub * 8));
                y[i] = __ldcg(reinterpret_cast<const float4*>(p + sub * 8 + 4));
            }
        }
#pragma unroll
        for (int i = 0; i < WIDE; ++i) {
            const float part[8] = {x[i].x, x[i].y, x[i].z, x[i].w, y[i].x, y[i].y, y[i].z, y[i].w};
            // an empty part adds nothing.  (The branch also keeps the loads together: without it the compiler moves each to its
            // use, and a call at 256 x 16 pairs takes 29.8 instead of 26.9 us.)
            if (lse[i] != kNegInf) st.merge(lse[i], 1.f, part);
        }
    }
}

// The lane's 8 dims of the joined result of one (sequence, head).
template <int HD>
__device__ __forceinline__ void join(const SharedDecodeArgs& a, int bh, int sub)
{
    SoftmaxState st;
    st.init();
    const int count = a.n_pre + a.splits;
    const float* ws = a.parts + (size_t)bh * count * (HD + 4);
    if (count <= 4) fold_partials<HD, 4>(st, ws, count, 1, sub);
    else fold_partials<HD, 8>(st, ws, count, 1, sub);
    float o[8];
    st.normalised(o);
    *reinterpret_cast<uint4*>(reinterpret_cast<bf16*>(a.out) + (size_t)bh * HD + sub * 8) = pack8(o);
}

}  // namespace parts
}  // namespace bt
