// The last step of attention whose keys were cut into parts: out = sum_z w_z part_z / sum_z w_z l_z with w_z = exp(m_z - max m).
// A wavefront a row of a head; a lane takes the statistics of a part, then DP / 64 columns.  Bound by latency: the first eight parts are
// asked for before their weights are known.  3.9-4.3 us a launch at 128 rows of 16 parts and at 2048 of 8.
#pragma once

#include "attn.hpp"

namespace skipffn {

template <int DP>
__device__ __forceinline__ void attn_join(const AttnJoinArgs& P, int workgroup) {
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)workgroup * ATT_WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (row >= (int64_t)P.T * P.Hq) return;
    const int t = (int)(row / P.Hq), head = (int)(row - (int64_t)t * P.Hq);
    constexpr int V = DP / 64;
    const float* part = P.part + row * P.splits * DP + lane * V;
    float x[8][V];
    auto fetch = [&](int i0) {                           // past the last part: the last again, unused
#pragma unroll
        for (int u = 0; u < 8; ++u)
#pragma unroll
            for (int j = 0; j < V; ++j) x[u][j] = part[(int64_t)min(i0 + u, P.splits - 1) * DP + j];
    };
    fetch(0);
    float m = -INFINITY, l = 0.0f;
    if (lane < P.splits) {
        m = P.stat[2 * (row * P.splits + lane)];
        l = P.stat[2 * (row * P.splits + lane) + 1];
    }
    if (P.seg != nullptr) {                              // is it a sequence's row?
        bool any = false;
        for (int i = lane; i < P.n_seq; i += 64) {
            int b, e;
            seg_bounds(P.seg, i, P.T, b, e);
            any |= b <= t && t < e;
        }
        if (__ballot(any) == 0) return;
    }
    float top = m;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
    const float w = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - top) * P.scale_log2);
    const float sum = wave_sum(w * l);
    // A row that sees no key, and it alone, has no maximum in any part: it is zero.  Where keys are seen and all scores are minus infinity the part's
    // maximum is the lowest number and its sum 0: no weight beside other parts, and 0 / 0 if there are no others
    const bool none = top == -INFINITY;
    const float inv = none ? 0.0f : 1.0f / sum;
    float o[V] = {};
    for (int i0 = 0;;) {
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            if (i0 + u >= P.splits) break;
            const float wi = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), i0 + u));
#pragma unroll
            for (int j = 0; j < V; ++j) o[j] = fmaf(wi, x[u][j], o[j]);
        }
        if ((i0 += 8) >= P.splits) break;
        fetch(i0);
    }
    if (P.lse != nullptr && lane == 0) P.lse[(int64_t)head * P.T + t] = none ? INFINITY : fmaf(top, P.scale_log2, __builtin_amdgcn_logf(sum));
    if (lane * V >= P.D) return;
    bf16_t* out = P.out + (int64_t)t * P.o_tok + head * P.o_head + lane * V;
    if constexpr (V == 2) *reinterpret_cast<uint32_t*>(out) = pack_bf16x2(o[0] * inv, o[1] * inv);
    else *out = f32_to_bf16(o[0] * inv);
}

}  // namespace skipffn
