// A cache cut down to the rows that received most: of every sequence and key/value head the n_keep rows of largest weight, where the `first` first and
// the `recent` last ones come before all others; equal weights by index, a NaN after every number.  The choice is unique for the weights given.
//
// Two kernels.  One workgroup a (sequence, head) finds the cut and writes the kept rows' numbers, ascending, and their weights.  Then the rows
// themselves: a lane takes 16 bytes of a row of k and of v, a workgroup 16 rows of a head (64 rows 51.6 us for 49.5 at 64 caches of 500 kept rows).
//
// The copy is bound by bytes: 8 heads of 128, 64 caches of up to 1000 rows to 500 49.5 us (236 MB, 4.8 TB/s), 4 of up to 32768 to 8000 53 (262 MB).  The
// search takes 9.5 and 25-27 us before it, the latter by the instructions of a compute unit a list: 4-5 us for each time over 32768 rows.
#include <algorithm>

#include "kernels.hpp"
#include "segments.hpp"

namespace skipffn {

// packed sequences whose offsets every workgroup finds by itself, a lane each; more take a kernel of their own (60 sequences of 616 rows 30.7 us so, 32.7 with it)
constexpr int EVICT_SCAN = 64;

// rows lo .. of sequence s and how many, how many of them stay, and the first of these among the rows that are kept
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
    if (P.n_seq > EVICT_SCAN) {                          // evict_offsets_kernel has been there
        q.to = P.seg_out[s];
        q.keep = P.seg_out[s + 1] - q.to;
        return q;
    }
    static_assert(EVICT_SCAN == 64, "a lane a sequence");
    const int lane = threadIdx.x & 63;
    int a = 0, b = 0;
    if (lane < P.n_seq) seg_bounds(P.seg, lane, P.T, a, b);
    const int mine = lane < P.n_seq ? evict_kept(P, lane, b - a) : 0;
    int64_t before = lane < s ? mine : 0;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) before += __shfl_xor(before, off, 64);
    q.to = (int)(before < P.T_out ? before : P.T_out);
    q.keep = min(evict_kept(P, s, q.n), P.T_out - q.to);
    return q;
}

// More than 64 packed sequences: where the kept rows of each begin, by one workgroup
__global__ __launch_bounds__(1024) void evict_offsets_kernel(const EvictArgs P) {
    __shared__ int64_t waves[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int64_t carry = 0;
    if (tid == 0) P.seg_out[0] = 0;
    for (int s0 = 0; s0 < P.n_seq; s0 += 1024) {
        int64_t v = 0;
        if (s0 + tid < P.n_seq) {
            int a, b;
            seg_bounds(P.seg, s0 + tid, P.T, a, b);
            v = evict_kept(P, s0 + tid, b - a);
        }
#pragma unroll
        for (int off = 1; off < 64; off *= 2) {
            const int64_t u = __shfl_up(v, off, 64);
            v += lane >= off ? u : 0;
        }
        __syncthreads();                                 // the last round's sums have been read
        if (lane == 63) waves[wave] = v;
        __syncthreads();
        int64_t all = 0;
        v += carry;
#pragma unroll
        for (int w = 0; w < 16; ++w) {
            v += w < wave ? waves[w] : 0;
            all += waves[w];
        }
        if (s0 + tid < P.n_seq) P.seg_out[s0 + tid + 1] = (int)(v < P.T_out ? v : P.T_out);
        carry += all;
    }
}

// The cut between what stays and what goes: the k smallest of a list's keys (rank_key) are those below `below`, and the first `ties` of those equal to it.
// Keys are counted by their first 11 bits (the sign, the exponent and two more, for weights), a prefix sum over the counts finds where the k-th lies, and
// those that share its bits are collected in LDS, where the next 11 and the last 10 bits are found the same way; in the list itself if they
// are too many.
struct EvictCut { uint32_t below; int ties; };
constexpr uint32_t EVICT_NONE = 0xFFFFFFFFu;             // key of a NaN
constexpr int EVICT_BINS = 2048, EVICT_CAND = 4096;
struct EvictShared {
    int hist[EVICT_BINS];
    uint32_t cand[EVICT_CAND];
    int waves[16], n_cand, bin, before, inside;
};
// rank_key<true> in fewer operations: with -0 made +0, a number that is not negative is turned round, a negative one increases already
__device__ __forceinline__ uint32_t evict_key(float v) {
    const uint32_t b = __float_as_uint(v + 0.0f), k = b ^ (~(uint32_t)((int32_t)b >> 31) >> 1);
    return v != v ? EVICT_NONE : k;
}
// The number with a key, or for a key that no number has one that compares as the key would: a NaN (no weight is at least that) before all numbers, minus
// infinity (every number is) after them
__device__ __forceinline__ float evict_number(uint32_t key) {
    return key > 0xFF800000u ? -INFINITY : __uint_as_float(key < 0x80000000u ? key ^ 0x7FFFFFFFu : key);
}
// for_keys(f) calls f with every key of the list that takes part, spread over the threads
template <int THREADS, class ForKeys>
__device__ __forceinline__ EvictCut evict_cut(ForKeys&& for_keys, int k, EvictShared& sh) {
    constexpr int WAVES = THREADS / 64, PER = EVICT_BINS / THREADS;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
#pragma unroll
    for (int i = 0; i < PER; ++i) sh.hist[tid + i * THREADS] = 0;
    if (tid == 0) sh.n_cand = 0;
    __syncthreads();
    for_keys([&](uint32_t v) { atomicAdd(&sh.hist[v >> 21], 1); });        // numbers end below bin 2047, which has the NaN
    uint32_t prefix = 0;                                 // the digits found so far
    bool in_lds = false;
    int cands = 0;
    for (int digit = 0;; ++digit) {
        const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0;
        if (digit > 0) {
            const uint32_t mask = 0xFFFFFFFFu << (digit == 1 ? 21 : 10), bits = digit == 1 ? EVICT_BINS - 1 : 1023;
            auto count = [&](uint32_t v) {
                if ((v & mask) == prefix) atomicAdd(&sh.hist[v >> shift & bits], 1);
            };
            if (in_lds) {
                for (int i = tid; i < cands; i += THREADS) count(sh.cand[i]);
            } else {
                for_keys(count);
            }
        }
        __syncthreads();
        int h[PER], mine = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            h[i] = sh.hist[PER * tid + i];
            sh.hist[PER * tid + i] = 0;                  // for the next digit
            mine += h[i];
        }
        const int incl = wave_inclusive_sum(mine);
        if (lane == 63) sh.waves[wave] = incl;
        __syncthreads();
        int before = incl - mine;
#pragma unroll
        for (int w = 0; w < WAVES - 1; ++w) before += w < wave ? sh.waves[w] : 0;
        if (before < k && k <= before + mine) {          // one thread
            int bin = 0, inside = h[0];
#pragma unroll
            for (int i = 1; i < PER; ++i)
                if (bin == i - 1 && k > before + inside) {
                    before += inside;
                    inside = h[i];
                    bin = i;
                }
            sh.bin = PER * tid + bin;
            sh.before = before;
            sh.inside = inside;
        }
        __syncthreads();
        if (digit == 0 && sh.bin == EVICT_BINS - 1) return EvictCut{EVICT_NONE, k - sh.before};       // all numbers, and the first of the others
        prefix |= (uint32_t)sh.bin << shift;
        if (k == sh.before + sh.inside) return EvictCut{prefix + (1u << shift), 0};       // numbers end below 2^32 - 2^22: no wrap
        k -= sh.before;
        if (digit == 2) return EvictCut{prefix, k};
        if (!in_lds && sh.inside <= EVICT_CAND) {        // uniform
            const uint32_t with = 0xFFFFFFFFu << shift;
            for_keys([&](uint32_t v) {
                if ((v & with) == prefix) sh.cand[atomicAdd(&sh.n_cand, 1)] = v;
            });
            cands = sh.inside;
            in_lds = true;
            __syncthreads();
        }
    }
}

// Weights of a list of n rows, four consecutive ones a load (and a thread); those past its end are any of it
typedef float f32x4_dword __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ f32x4 four_weights(const float* w, int t, int n) {
    if (n < 4) return f32x4{w[min(t, n - 1)], w[min(t + 1, n - 1)], w[min(t + 2, n - 1)], w[min(t + 3, n - 1)]};      // uniform
    // the last rows are read with those before them, and moved up
    const int at = min(t, n - 4), up = t - at;
    f32x4 v = *reinterpret_cast<const f32x4_dword*>(w + at);
    if (__ballot(up != 0) != 0) {
        v[0] = up == 1 ? v[1] : up == 2 ? v[2] : up == 3 ? v[3] : v[0];
        v[1] = up == 1 ? v[2] : up == 2 ? v[3] : v[1];
        v[2] = up == 1 ? v[3] : v[2];
    }
    return v;
}

// A list of up to 4 THREADS rows is read once and lies in registers.  A longer one is read again for every step, some loads of a thread under way at a time (a
// compute unit's share of a list's bytes is bound by latency).  For the kept rows a wavefront has a range of them: it counts those that stay and those equal
// to the cut, and when the counts of the wavefronts before it are known goes over them again and writes, without a barrier in between.
template <int THREADS, bool LONG>
__global__ __launch_bounds__(THREADS) void evict_select_kernel(const EvictArgs P) {
    constexpr int WAVES = THREADS / 64, AHEAD = LONG ? 4 : 1;
    __shared__ EvictShared sh;
    __shared__ int counts[WAVES][2];                     // below the cut, equal to it
    const int s = (int)blockIdx.x / P.Hkv, head = (int)blockIdx.x % P.Hkv, tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const EvictSeq q = evict_seq(P, s);
    if (head == 0 && tid == 0 && (!P.packed || P.n_seq <= EVICT_SCAN)) {
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
    const int n = q.n;
    // rows that stay before all others: [0, first) and [recent, n)
    const int first = min(P.first, n), recent = max(n - P.recent, first), stay = first + n - recent;
    const bool in_regs = !LONG || n <= 4 * THREADS;      // uniform
    const f32x4 mine = four_weights(w, 4 * tid, n);
    EvictCut cut{0, 0};                                  // of the rows that do not stay anyway
    bool among_stay = false;                             // `ties` rows of those that stay are all that is kept
    auto give = [&](auto&& f, const f32x4& v, int t) {
        const int t0 = __builtin_amdgcn_readfirstlane(t);           // of the wavefront's 256 rows
        if (t0 >= first && t0 + 256 <= recent) {
#pragma unroll
            for (int j = 0; j < 4; ++j) f(evict_key(v[j]));
        } else if (t0 < recent && t0 + 256 > first) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (t + j >= first && t + j < recent) f(evict_key(v[j]));
        }
    };
    if (q.keep >= n) {
        cut = EvictCut{EVICT_NONE, n};
    } else if (q.keep <= stay) {
        among_stay = true;
        cut.ties = q.keep;
    } else {
        cut = evict_cut<THREADS>([&](auto&& f) {
            if (in_regs) {
                give(f, mine, 4 * tid);
                return;
            }
            for (int t = 4 * tid; t < recent; t += 4 * AHEAD * THREADS) {
                f32x4 v[AHEAD];
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) v[i] = four_weights(w, t + i * 4 * THREADS, n);
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) give(f, v[i], t + i * 4 * THREADS);
            }
        }, q.keep - stay, sh);
    }
    // The wavefront's rows, 256 at a time: f(weights, the lane's first row)
    const int blocks = (n + 255) / 256, b0 = in_regs ? wave : blocks * wave / WAVES, b1 = in_regs ? min(wave + 1, blocks) : blocks * (wave + 1) / WAVES;
    auto for_rows = [&](auto&& f) {
        if (in_regs) {
            if (b0 < b1) f(mine, 4 * tid);
            return;
        }
        for (int b = b0; b < b1; b += AHEAD) {
            f32x4 v[AHEAD];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) v[i] = four_weights(w, (b + i) * 256 + 4 * lane, n);
#pragma unroll
            for (int i = 0; i < AHEAD; ++i)
                if (b + i < b1) f(v[i], (b + i) * 256 + 4 * lane);
        }
    };
    // The cut as comparisons of weights, whose order is that of their keys: kept are those not below `least`, and ties are equal to `tie`
    const float least = among_stay ? NAN : evict_number(cut.below - 1), tie = evict_number(cut.below);
    const bool ties = cut.ties > 0, tie_nan = cut.below == EVICT_NONE;       // uniform
    // flags of four rows, those kept below the cut and ties
    auto flags = [&](const f32x4& x, int t, bool (&below)[4], bool (&equal)[4]) {
        const int t0 = __builtin_amdgcn_readfirstlane(t);
        const bool inside = t0 >= first && t0 + 256 <= recent;               // uniform
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            below[j] = x[j] >= least;
            equal[j] = tie_nan ? x[j] != x[j] : x[j] == tie;
        }
        if (among_stay || !inside) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool in = t + j < n, must = t + j < first || t + j >= recent;
                below[j] = in && !among_stay && (must || below[j]);
                equal[j] = in && (among_stay ? must : !must && equal[j]);
            }
        }
    };
    int below = 0, equal = 0;
    for_rows([&](const f32x4& x, int t) {
        bool fb[4], fe[4];
        flags(x, t, fb, fe);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            below += __popcll(__ballot(fb[j]));
            if (ties) equal += __popcll(__ballot(fe[j]));
        }
    });
    if (lane == 0) {
        counts[wave][0] = below;
        counts[wave][1] = equal;
    }
    __syncthreads();
    int at = 0, ties_before = 0;                         // kept rows and ties of the wavefronts before this one
    for (int i = 0; i < wave; ++i) {
        at += counts[i][0] + min(max(cut.ties - ties_before, 0), counts[i][1]);
        ties_before += counts[i][1];
    }
    for_rows([&](const f32x4& x, int t) {
        bool kept[4], fe[4];
        flags(x, t, kept, fe);
        if (ties) {
            int tie_at = ties_before;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint64_t m = __ballot(fe[j]);
                tie_at += lanes_below(m);
                ties_before += __popcll(m);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) kept[j] = kept[j] || (fe[j] && tie_at++ < cut.ties);
        }
        int to = at;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint64_t m = __ballot(kept[j]);
            to += lanes_below(m);
            at += __popcll(m);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (kept[j]) {
                keep[to] = t + j;
                if (w_out != nullptr) w_out[to] = x[j];
                ++to;
            }
    });
}

// Where no list can have more than 2048 rows a form of 512 threads that holds four a thread, otherwise one of 1024 that reads lists of more than 4096 again (us of whole calls, 512
// threads / the other form: 512 lists of 300 rows 19.3 / 23.9, of up to 1000 58.4 / 63.7).  512 lists of 4000 take 123.1, by a form of 1024 threads that only holds them 122.9: there is none
constexpr int EVICT_ROWS = 16, EVICT_THREADS = 256, EVICT_SHORT = 2048, EVICT_LONG_THREADS = 1024;

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
    return std::max<int64_t>((int64_t)a.n_seq * a.Hkv * (EVICT_LONG_THREADS / EVICT_THREADS), gather_chunks(a) * (a.packed ? 1 : a.n_seq) * a.Hkv);
}

hipError_t launch_evict(const EvictArgs& a, hipStream_t s) {
    const uint32_t lists = (uint32_t)(a.n_seq * a.Hkv);
    if (a.packed && a.n_seq > EVICT_SCAN) evict_offsets_kernel<<<1, 1024, 0, s>>>(a);
    if (a.T <= EVICT_SHORT) evict_select_kernel<EVICT_SHORT / 4, false><<<lists, EVICT_SHORT / 4, 0, s>>>(a);
    else evict_select_kernel<EVICT_LONG_THREADS, true><<<lists, EVICT_LONG_THREADS, 0, s>>>(a);
    const hipError_t e = hipGetLastError();
    const int64_t chunks = gather_chunks(a), wgs = chunks * (a.packed ? 1 : a.n_seq) * a.Hkv;
    if (e != hipSuccess || wgs == 0) return e;
    evict_gather_kernel<<<(uint32_t)wgs, EVICT_THREADS, 0, s>>>(a, (int)chunks);
    return hipGetLastError();
}

}  // namespace skipffn
