// What the rows of a cache receive from single tokens: w[kv head][t] = sum over the rows of a product (sequence, query head) that see t of
// 2^(c s - lse), s the products that the attention left in the workspace, lse its rows' log-sum-exps.  A thread owns a row of the cache; the products
// of a (sequence, head) lie along the cache's rows, so that a wavefront reads 256 bytes of them at a time.  Where many sequences share a prefix
// the wavefronts of a workgroup take a part of them each for the same 64 rows, and are joined in order.
//
// Bound by the products' bytes: 4 Hq a row of the cache, where its keys and values are 4 Hkv D.
#include "kernels.hpp"
#include "segments.hpp"

namespace skipffn {

constexpr int DW_THREADS = 256;

template <int WAYS>                                      // wavefronts that share the sequences of 256 / WAYS cache rows
__global__ __launch_bounds__(DW_THREADS) void decode_weights_kernel(const AttnDecodeArgs P, const DecodeWeightsArgs W, const int prefix_chunks) {
    constexpr int CH = DW_THREADS / WAYS;
    const int g = P.Hq / P.Hkv, kvh = (int)blockIdx.x % P.Hkv, chunk = (int)blockIdx.x / P.Hkv;
    const float c = P.scale_log2;
    if (chunk < prefix_chunks) {
        int group, t0, nt;
        if (!locate_chunk<CH, false>(P.prefix_seg, P.n_groups, P.Tp, chunk, group, t0, nt)) return;
        int lo, hi;
        seg_bounds(P.group_off, group, P.n_seq, lo, hi);
        const int rows = min(hi - lo, P.most_shared) * g;
        const int way = (int)threadIdx.x / CH, t = (int)threadIdx.x % CH;
        const bool in = t < nt;
        const float* s = P.prefix_scores + (int64_t)kvh * P.most_shared * g * P.Tp + t0 + (in ? t : 0);
        const int i0 = rows * way / WAYS, i1 = rows * (way + 1) / WAYS;
        float sum = 0.0f;
#pragma unroll 8
        for (int i = i0; i < i1; ++i) {
            const float lse = P.lse[(int64_t)(kvh * g + i % g) * P.n_seq + lo + i / g];
            sum += __builtin_amdgcn_exp2f(fmaf(s[(int64_t)i * P.Tp], c, -lse));
        }
        if constexpr (WAYS > 1) {
            __shared__ float parts[WAYS][CH];
            parts[way][t] = sum;
            __syncthreads();
            if (way > 0) return;
            sum = 0.0f;
#pragma unroll
            for (int i = 0; i < WAYS; ++i) sum += parts[i][t];
        }
        if (!in) return;
        float* w = W.prefix_w + kvh * W.prefix_head + t0 + t;
        *w = W.accumulate ? *w + sum : sum;
        return;
    }
    const int own_chunks = (P.cap + DW_THREADS - 1) / DW_THREADS, q = chunk - prefix_chunks;
    const int seq = q / own_chunks, t = q % own_chunks * DW_THREADS + (int)threadIdx.x;
    if (t >= min(max(P.suffix_len[seq], 0), P.cap)) return;
    float sum = 0.0f;
    for (int e = 0; e < g; ++e) {
        const int head = kvh * g + e;
        sum += __builtin_amdgcn_exp2f(fmaf(P.own_scores[((int64_t)seq * P.Hq + head) * P.cap + t], c, -P.lse[(int64_t)head * P.n_seq + seq]));
    }
    float* w = W.own_w + seq * W.own_seq + kvh * W.own_head + t;
    *w = W.accumulate ? *w + sum : sum;
}

namespace {
int weight_ways(const AttnDecodeArgs& a) { return (int64_t)a.most_shared * (a.Hq / a.Hkv) > 16 ? 4 : 1; }
int64_t prefix_chunks_of(const AttnDecodeArgs& a) {
    const int64_t ch = DW_THREADS / weight_ways(a);
    return a.Tp > 0 ? (a.Tp + ch - 1) / ch + a.n_groups : 0;
}
}  // namespace

int64_t decode_weights_workgroups(const AttnDecodeArgs& a) {
    return (prefix_chunks_of(a) + (int64_t)a.n_seq * ((a.cap + DW_THREADS - 1) / DW_THREADS)) * a.Hkv;
}

hipError_t launch_decode_weights(const AttnDecodeArgs& a, const DecodeWeightsArgs& w, hipStream_t s) {
    const uint32_t grid = (uint32_t)decode_weights_workgroups(a);
    if (grid == 0) return hipSuccess;
    if (weight_ways(a) == 1) decode_weights_kernel<1><<<grid, DW_THREADS, 0, s>>>(a, w, (int)prefix_chunks_of(a));
    else decode_weights_kernel<4><<<grid, DW_THREADS, 0, s>>>(a, w, (int)prefix_chunks_of(a));
    return hipGetLastError();
}

}  // namespace skipffn
