// A cache cut down to the rows that received most: of every sequence and key/value head the n_keep rows of largest weight, where the `first` first and
// the `recent` last ones come before all others; equal weights by index, a NaN after every number.  The choice is unique for the weights given.
//
// Two kernels.  One workgroup a (sequence, head) finds the cut (topk.hpp; the keys stay in registers up to 64 a thread, longer lists are read again from
// L2 for every step) and writes the kept rows' numbers, ascending, and their weights.  Then the rows themselves: a lane takes 16 bytes of a row of
// k and of v, a workgroup 64 rows of a head.
#include <algorithm>

#include "kernels.hpp"
#include "segments.hpp"
#include "topk.hpp"

namespace skipffn {

// rows [lo, hi) of sequence s, how many of them stay, and the first of these among the rows that are kept
struct EvictSeq { int lo, n, keep, to; };
__device__ __forceinline__ int evict_kept(const EvictArgs& P, int s, int n) {
    return min(max(P.n_keep_dev != nullptr ? P.n_keep_dev[s] : P.n_keep, 0), n);
}
__device__ __forceinline__ EvictSeq evict_seq(const EvictArgs& P, int s) {
    EvictSeq q{0, 0, 0, 0};
    if (!P.packed) {
        q.n = min(max(P.seg[s], 0), P.T);
        q.keep = min(evict_kept(P, s, q.n), P.T_out);
        return q;
    }
    int hi;
    seg_bounds(P.seg, s, P.T, q.lo, hi);
    q.n = hi - q.lo;
    const int lane = threadIdx.x & 63;
    int64_t before = 0;
    for (int i = lane; i < s; i += 64) {
        int a, b;
        seg_bounds(P.seg, i, P.T, a, b);
        before += evict_kept(P, i, b - a);
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) before += __shfl_xor(before, off, 64);
    q.to = (int)(before < P.T_out ? before : P.T_out);
    q.keep = min(evict_kept(P, s, q.n), P.T_out - q.to);
    return q;
}

constexpr int EVICT_MAXV = 64;                           // keys of a thread that stay in registers

// MAXV > 0: lists of up to MAXV * 1024 rows in registers; LONG: longer ones too
template <int MAXV, bool LONG>
__global__ __launch_bounds__(TOPK_THREADS) void evict_select_kernel(const EvictArgs P) {
    __shared__ TopkShared sh;
    __shared__ int counts[MAXV * TOPK_WAVES];
    const int s = (int)blockIdx.x / P.Hkv, head = (int)blockIdx.x % P.Hkv, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const EvictSeq q = evict_seq(P, s);
    if (head == 0 && tid == 0) {
        if (P.packed) {
            P.seg_out[s + 1] = q.to + q.keep;
            if (s == 0) P.seg_out[0] = 0;
        } else {
            P.seg_out[s] = q.keep;
        }
    }
    if (q.keep == 0) return;
    const float* w = P.w + (P.packed ? 0 : s * P.w_seq) + head * P.w_head + q.lo;
    float* w_out = P.w_out == nullptr ? nullptr : P.w_out + (P.packed ? 0 : s * P.wo_seq) + head * P.wo_head + q.to;
    int32_t* keep = P.keep + (P.packed ? 0 : s * P.keep_seq) + head * P.keep_head + q.to;
    const int n = q.n, nv = (n + TOPK_THREADS - 1) / TOPK_THREADS;
    auto key_of = [&](int t) { return t >= n ? TOPK_NONE : t < P.first || t >= n - P.recent ? 0u : rank_key<true>(w[t]); };
    const bool all = q.keep >= n;                        // uniform
    auto put = [&](int at, int t) {
        keep[at] = t;
        if (w_out != nullptr) w_out[at] = w[t];
    };
    if (!LONG || nv <= MAXV) {
        uint32_t key[MAXV];
        // before[i]: entries flagged before entry i * 1024 + tid; every wavefront's counts go through LDS
        auto prefix = [&](auto&& flag, int (&before)[MAXV]) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < MAXV; ++i)
                if (i < nv) {
                    const uint64_t m = __ballot(flag(i));
                    before[i] = lanes_below(m);
                    if (lane == 0) counts[i * TOPK_WAVES + wave] = __popcll(m);
                }
            __syncthreads();
            if (wave == 0) {
                int carry = 0;
                for (int c = 0; c < nv * TOPK_WAVES; c += 64) {
                    const bool in = c + lane < nv * TOPK_WAVES;
                    const int v = in ? counts[c + lane] : 0, incl = wave_inclusive_sum(v);
                    if (in) counts[c + lane] = carry + incl - v;
                    carry += __builtin_amdgcn_readlane(incl, 63);
                }
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < MAXV; ++i)
                if (i < nv) before[i] += counts[i * TOPK_WAVES + wave];
        };
#pragma unroll
        for (int i = 0; i < MAXV; ++i)
            if (i < nv) key[i] = key_of(i * TOPK_THREADS + tid);
        TopkCut cut{TOPK_NONE, n};                       // everything: every key <= NONE
        if (!all) cut = topk_cut<MAXV>([&](int i) { return key[i]; }, nv, q.keep, sh);
        int before[MAXV];
        uint64_t kept = 0;                               // bit i: entry i of the thread
        if (cut.ties > 0 && !all) {
            prefix([&](int i) { return key[i] == cut.cut && i * TOPK_THREADS + tid < n; }, before);
#pragma unroll
            for (int i = 0; i < MAXV; ++i)
                if (i < nv && key[i] == cut.cut && before[i] < cut.ties) kept |= (uint64_t)1 << i;
        }
#pragma unroll
        for (int i = 0; i < MAXV; ++i)
            if (i < nv && (key[i] < cut.cut || (all && i * TOPK_THREADS + tid < n))) kept |= (uint64_t)1 << i;
#pragma unroll
        for (int i = 0; i < MAXV; ++i)
            if (i < nv && i * TOPK_THREADS + tid >= n) kept &= ~((uint64_t)1 << i);
        prefix([&](int i) { return (kept >> i & 1) != 0; }, before);
#pragma unroll
        for (int i = 0; i < MAXV; ++i)
            if (i < nv && (kept >> i & 1) != 0) put(before[i], i * TOPK_THREADS + tid);
        return;
    }
    if constexpr (LONG) {
        TopkCut cut{TOPK_NONE, n};
        if (!all) cut = topk_cut<0>([&](int i) { return key_of(i * TOPK_THREADS + tid); }, nv, q.keep, sh);
        int ties_before = 0, kept_before = 0;
        for (int i = 0; i < nv; ++i) {
            const int t = i * TOPK_THREADS + tid;
            const uint32_t key = key_of(t);
            int before[1] = {0};
            if (cut.ties > 0 && !all) {
                const int here = topk_prefix<1>([&](int) { return key == cut.cut && t < n; }, 1, sh, before);
                before[0] += ties_before;
                ties_before += here;
            }
            const bool in = t < n && (all || key < cut.cut || (key == cut.cut && before[0] < cut.ties));
            const int here = topk_prefix<1>([&](int) { return in; }, 1, sh, before);
            if (in) put(kept_before + before[0], t);
            kept_before += here;
        }
    }
}

constexpr int EVICT_ROWS = 64, EVICT_THREADS = 256;

__global__ __launch_bounds__(EVICT_THREADS) void evict_gather_kernel(const EvictArgs P, const int chunks) {
    const int head = (int)blockIdx.x % P.Hkv, q = (int)blockIdx.x / P.Hkv;
    int s, r0, rows, lo = 0;
    if (P.packed) {
        if (!locate_chunk<EVICT_ROWS, false>(P.seg_out, P.n_seq, P.T_out, q, s, r0, rows)) return;
        int hi;
        seg_bounds(P.seg, s, P.T, lo, hi);
    } else {
        s = q / chunks;
        r0 = q % chunks * EVICT_ROWS;
        rows = min(min(P.seg_out[s], P.T_out) - r0, EVICT_ROWS);
        if (rows <= 0) return;
    }
    const int64_t sq = P.packed ? 0 : s;
    const bf16_t* k = P.k.p + sq * P.k_seq + head * P.k.head;
    const bf16_t* v = P.v.p + sq * P.v_seq + head * P.v.head;
    bf16_t* ko = P.k_out.p + sq * P.ko_seq + head * P.k_out.head;
    bf16_t* vo = P.v_out.p + sq * P.vo_seq + head * P.v_out.head;
    const int32_t* keep = P.keep + sq * P.keep_seq + head * P.keep_head;
    const int per_row = P.D / 8;
    for (int i = threadIdx.x; i < rows * per_row; i += EVICT_THREADS) {
        const int r = r0 + i / per_row, c = i % per_row * 8;
        const int64_t from = lo + keep[r];
        const u32x4 a = *reinterpret_cast<const u32x4*>(k + from * P.k.tok + c), b = *reinterpret_cast<const u32x4*>(v + from * P.v.tok + c);
        *reinterpret_cast<u32x4*>(ko + (int64_t)r * P.k_out.tok + c) = a;
        *reinterpret_cast<u32x4*>(vo + (int64_t)r * P.v_out.tok + c) = b;
    }
}

namespace {
int64_t gather_chunks(const EvictArgs& a) {
    if (a.packed) return ((int64_t)a.T_out + EVICT_ROWS - 1) / EVICT_ROWS + a.n_seq;
    return ((int64_t)(a.n_keep_dev != nullptr ? a.T_out : std::min(a.T_out, a.n_keep)) + EVICT_ROWS - 1) / EVICT_ROWS;
}
}  // namespace

int64_t evict_workgroups(const EvictArgs& a) {
    return std::max<int64_t>((int64_t)a.n_seq * a.Hkv * (TOPK_THREADS / EVICT_THREADS), gather_chunks(a) * (a.packed ? 1 : a.n_seq) * a.Hkv);
}

hipError_t launch_evict(const EvictArgs& a, hipStream_t s) {
    const dim3 grid((uint32_t)(a.n_seq * a.Hkv));
    if (a.T <= 4 * TOPK_THREADS) evict_select_kernel<4, false><<<grid, TOPK_THREADS, 0, s>>>(a);
    else if (a.T <= 16 * TOPK_THREADS) evict_select_kernel<16, false><<<grid, TOPK_THREADS, 0, s>>>(a);
    else if (a.T <= EVICT_MAXV * TOPK_THREADS) evict_select_kernel<EVICT_MAXV, false><<<grid, TOPK_THREADS, 0, s>>>(a);
    else evict_select_kernel<EVICT_MAXV, true><<<grid, TOPK_THREADS, 0, s>>>(a);
    const hipError_t e = hipGetLastError();
    const int64_t chunks = gather_chunks(a), wgs = chunks * (a.packed ? 1 : a.n_seq) * a.Hkv;
    if (e != hipSuccess || wgs == 0) return e;
    evict_gather_kernel<<<(uint32_t)wgs, EVICT_THREADS, 0, s>>>(a, (int)chunks);
    return hipGetLastError();
}

}  // namespace skipffn
