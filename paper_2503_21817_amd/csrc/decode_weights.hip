// What the rows of a cache receive from single tokens: w[kv head][t] = sum over the rows of a product (sequence, query head) that see t of
// 2^(c s - lse), s the products that the attention left in the workspace, lse its rows' log-sum-exps, here from the statistics of the parts
// that the keys were cut into; the first workgroups join those parts' rows (attn_join.hpp).  A thread owns a row of the cache; the products of a
// (sequence, head) lie along the cache's rows, so that a wavefront reads 256 bytes of them at a time.  Where many sequences share a prefix the
// wavefronts of a workgroup take a part of them each for the same 64 rows, and are joined in order.
//
// 4 caches of up to 32768 rows (32 / 8 heads: 10 MB of products) 8.4 us, a chain of loads: bounds, statistics, products; 64 sequences on two prefixes of up to 5795 rows
// (36 MB) 10.  Join and weights in kernels of their own took 4.7 + 7.6 and 4.7 + 6.6 and a launch more.
#include "attn_join.hpp"

namespace skipffn {

constexpr int DW_THREADS = ATT_THREADS;

// Log-sum-exps of up to DW_THREADS rows into LDS, row r that of query head head(r) of sequence seq(r): with parts, some lanes a row, a part each
template <class Row>
__device__ __forceinline__ void rows_lse(const AttnDecodeArgs& P, int rows, const Row& row, float* lse) {
    if (P.splits == 1) {
        for (int r = threadIdx.x; r < rows; r += DW_THREADS) {
            const int2 at = row(r);
            lse[r] = P.lse[(int64_t)at.y * P.n_seq + at.x];
        }
        return;
    }
    int lanes = 2;
    while (lanes < P.splits) lanes *= 2;                 // 64 at most
    const int part = (int)threadIdx.x % lanes;
    for (int r = (int)threadIdx.x / lanes; r < rows; r += DW_THREADS / lanes) {
        const int2 at = row(r);
        const float* stat = P.stat + 2 * (((int64_t)at.x * P.Hq + at.y) * P.splits + min(part, P.splits - 1));
        const float m = part < P.splits ? stat[0] : -INFINITY, l = stat[1];
        float top = m;
        for (int off = lanes / 2; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
        float sum = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - top) * P.scale_log2) * l;
        for (int off = lanes / 2; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
        if (part == 0) lse[r] = top == -INFINITY ? INFINITY : fmaf(top, P.scale_log2, __builtin_amdgcn_logf(sum));
    }
}

template <int DP, int WAYS>                              // wavefronts that share the sequences of 256 / WAYS cache rows
__global__ __launch_bounds__(DW_THREADS) void decode_weights_kernel(const AttnDecodeArgs P, const DecodeWeightsArgs W, const AttnJoinArgs J,
                                                                    const int joins, const int prefix_chunks) {
    constexpr int CH = DW_THREADS / WAYS;
    __shared__ float lse[DW_THREADS];
    if ((int)blockIdx.x < joins) {
        attn_join<DP>(J, (int)blockIdx.x);
        return;
    }
    const int wg = (int)blockIdx.x - joins, g = P.Hq / P.Hkv, kvh = wg % P.Hkv, chunk = wg / P.Hkv;
    const float c = P.scale_log2;
    if (chunk < prefix_chunks) {
        int group, t0, nt;
        if (!locate_chunk<CH, false>(P.prefix_seg, P.n_groups, P.Tp, chunk, group, t0, nt)) return;
        int lo, hi;
        seg_bounds(P.group_off, group, P.n_seq, lo, hi);
        const int rows = min(hi - lo, P.most_shared) * g;
        const int way = (int)threadIdx.x / CH, t = (int)threadIdx.x % CH;
        const bool in = t < nt;
        int p0, p1;
        seg_bounds(P.prefix_seg, group, P.Tp, p0, p1);
        const float* s = P.prefix_scores + (int64_t)kvh * P.most_shared * g * P.prefix_ld + decode_score_at(p0, group) + t0 - p0 + (in ? t : 0);
        float sum = 0.0f;
        for (int r0 = 0; r0 < rows; r0 += DW_THREADS) {
            const int n = min(rows - r0, DW_THREADS), i0 = n * way / WAYS, i1 = n * (way + 1) / WAYS;
            float x[4];                                  // the first products come with the rows' statistics
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = s[(int64_t)(r0 + min(i0 + i, n - 1)) * P.prefix_ld];
            __syncthreads();                             // the last ones have been read
            rows_lse(P, n, [&](int r) { return int2{lo + (r0 + r) / g, kvh * g + (r0 + r) % g}; }, lse);
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 4; ++i) sum += i0 + i < i1 ? __builtin_amdgcn_exp2f(fmaf(x[i], c, -lse[i0 + i])) : 0.0f;
#pragma unroll 8
            for (int i = i0 + 4; i < i1; ++i) sum += __builtin_amdgcn_exp2f(fmaf(s[(int64_t)(r0 + i) * P.prefix_ld], c, -lse[i]));
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
    const int seq = q / own_chunks, t0 = q % own_chunks * DW_THREADS, t = t0 + (int)threadIdx.x, own = min(max(P.suffix_len[seq], 0), P.cap);
    if (t0 >= own) return;
    const float* s = P.own_scores + ((int64_t)seq * P.Hq + kvh * g) * P.own_ld + min(t, own - 1);
    float sum = 0.0f;
    for (int r0 = 0; r0 < g; r0 += DW_THREADS) {
        const int n = min(g - r0, DW_THREADS);
        __syncthreads();
        rows_lse(P, n, [&](int r) { return int2{seq, kvh * g + r0 + r}; }, lse);
        __syncthreads();
#pragma unroll 4
        for (int i = 0; i < n; ++i) sum += __builtin_amdgcn_exp2f(fmaf(s[(int64_t)(r0 + i) * P.own_ld], c, -lse[i]));
    }
    if (t >= own) return;
    float* w = W.own_w + seq * W.own_seq + kvh * W.own_head + t;
    *w = W.accumulate ? *w + sum : sum;
}

namespace {
int64_t prefix_chunks_of(const AttnDecodeArgs& a) {
    const int64_t ch = DW_THREADS / a.ways;
    return a.Tp > 0 ? (a.Tp + ch - 1) / ch + a.n_groups : 0;
}
int64_t joins_of(const AttnDecodeArgs& a) { return a.splits > 1 ? ((int64_t)a.n_seq * a.Hq + ATT_WAVES - 1) / ATT_WAVES : 0; }
}  // namespace

// Four wavefronts a shared row where one leaves compute units without work (32 / 8 heads, us of whole calls, one / four; products of a row beside its rows):
//     rows      8              16             32             64             128
//      1500   12.3 / 12.1    13.9 / 13.2    17.0 / 16.3    23.5 / 22.0    30.9 / 26.7
//      4000   15.2 / 15.0    18.1 / 17.5    19.3 / 19.2    27.0 / 25.7    33.8 / 30.5
//      8000   19.4 / 19.9    26.1 / 26.1    27.1 / 28.5    32.9 / 33.1    51.1 / 47.9
//     16000   25.2 / 26.3    28.3 / 29.4    38.7 / 42.0    47.8 / 50.2    74.7 / 74.6
//     24000   36.0 / 39.0    42.7 / 46.6    53.2 / 61.2    73.0 / 79.0   110.3 / 113.5
int decode_weight_ways(int64_t Tp, int64_t Hq, int64_t Hkv, int64_t most_shared, int ncu) {
    const int64_t products = most_shared * (Hq / Hkv), blocks = Tp / DW_THREADS * Hkv;
    return products >= 8 && blocks <= (products > 64 ? ncu : ncu / 2) ? 4 : 1;
}

int64_t decode_weights_workgroups(const AttnDecodeArgs& a) {
    return joins_of(a) + (prefix_chunks_of(a) + (int64_t)a.n_seq * ((a.cap + DW_THREADS - 1) / DW_THREADS)) * a.Hkv;
}

template <int DP>
static void launch_dw(const AttnDecodeArgs& a, const DecodeWeightsArgs& w, const AttnJoinArgs& j, uint32_t grid, hipStream_t s) {
    if (a.ways == 1) decode_weights_kernel<DP, 1><<<grid, DW_THREADS, 0, s>>>(a, w, j, (int)joins_of(a), (int)prefix_chunks_of(a));
    else decode_weights_kernel<DP, 4><<<grid, DW_THREADS, 0, s>>>(a, w, j, (int)joins_of(a), (int)prefix_chunks_of(a));
}

hipError_t launch_decode_weights(const AttnDecodeArgs& a, const DecodeWeightsArgs& w, const AttnJoinArgs& j, hipStream_t s) {
    const uint32_t grid = (uint32_t)decode_weights_workgroups(a);
    if (grid == 0) return hipSuccess;
    if (a.D <= 64) launch_dw<64>(a, w, j, grid, s);
    else launch_dw<128>(a, w, j, grid, s);
    return hipGetLastError();
}

}  // namespace skipffn
