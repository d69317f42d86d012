// Attention of packed sequences on v_mfma_f32_32x32x16_bf16: what the forward, the backward and the single-token kernels share.
//
// With S = scale Q K^T over the keys a row sees, P = softmax(S) by rows and O = P V.  Every product is taken with the result
// transposed so that the exponentials a lane computes are already an operand of the next product:
//   S^T [key][query] = K Q^T    leaves a lane one query (column lane % 32) and 16 of 32 keys (8 (i / 4) + 4 (lane / 32) + i % 4);
//   O^T [d][query] = V^T P^T    takes the same registers, rounded to bf16, as its second operand: the order of the contraction is
//                               free, so V^T is read in the order of keys that the lane holds.
// Row maxima and sums then stay inside a lane but for one exchange with the lane 32 further.
//
// A kernel for 64, 96 or 128 columns serves heads of up to as many.  A tile of rows [token][column] of one head lies in LDS with
// 128 bytes a row (64 columns) or 256, 16-byte chunk c of row r at c ^ tile_swz(r).  The same placing serves both ways it is read,
// free of bank conflicts: 16 consecutive rows at one chunk (ds_read_b128, the operand whose contraction runs along the columns) and
// 4 rows x 64 bytes (ds_read_b64_tr_b16, the operand whose contraction runs along the tokens).
#pragma once

#include <cfloat>

#include "kernels.hpp"
#include "segments.hpp"

namespace skipffn {

constexpr int ATT_ROWS = 32;               // queries of a wavefront
constexpr int ATT_WAVES = 4;
constexpr int ATT_THREADS = ATT_WAVES * 64;

typedef __attribute__((address_space(3))) bf16x4* lds_bf16x4_ptr;

// ---- tiles in LDS ----------------------------------------------------------------------------------
template <int DP> constexpr int tile_row_bytes() { return DP <= 64 ? 128 : 256; }
template <int DP>
__device__ __forceinline__ int tile_swz(int r) {
    return DP <= 64 ? (((r >> 1) & 1) << 2) | ((r >> 2) & 3) : ((r & 3) << 2) | ((r >> 2) & 3);
}
template <int DP>
__device__ __forceinline__ uint32_t tile_off(int r, int chunk) {
    return (uint32_t)(r * tile_row_bytes<DP>() + ((chunk ^ tile_swz<DP>(r)) << 4));
}

// The rows of one head of one sequence: row r at base + r * stride elements
struct HeadRows { const bf16_t* base; int stride; };

// A tile of N rows on its way through registers: issued as buffer loads, stored to LDS a tile later.  Columns at and past the head's read
// zeros, and so do rows at and past `rows` where rows are apart.  With a stride of less than a row's columns (0: every row is the same one) the last
// row lies where they do and they read of it: never what is not the head's in this sequence, but they have to be masked by who uses them.
template <int DP, int N, int THREADS = ATT_THREADS>
struct TileLoad {
    static constexpr int CH = tile_row_bytes<DP>() / 16;        // 16-byte chunks of a row in LDS
    static constexpr int PER = N * CH / THREADS;
    static_assert(N * CH % THREADS == 0, "whole rows");
    u32x4 v[PER];
    // byte offset of the thread's first chunk, or none for a chunk past the head's columns; the next ones are THREADS / CH rows on
    static __device__ __forceinline__ uint32_t first(int tid, int stride, int D) {
        const int c = tid % CH;
        return c * 8 < D ? (uint32_t)((tid / CH) * stride + c * 8) * 2u : kOobOffset;
    }
    __device__ __forceinline__ void load(const HeadRows& h, int row0, int rows, int D, uint32_t off) {
        const int n = rows - row0 < N ? rows - row0 : N;
        const __amdgpu_buffer_rsrc_t r =
            make_rsrc(h.base + (int64_t)row0 * h.stride, n > 0 ? (uint32_t)((n - 1) * h.stride + D) * 2u : 0u);
#pragma unroll
        for (int i = 0; i < PER; ++i)
            v[i] = __builtin_amdgcn_raw_buffer_load_b128(r, (int)(off + (uint32_t)(i * (THREADS / CH) * h.stride) * 2u), 0, 0);
    }
    // whether the thread holds an infinity or a NaN: an exponent of ones, the largest of all as unsigned 16-bit halves
    __device__ __forceinline__ bool any_not_finite() const {
        typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
        u16x2 top = {0, 0};
#pragma unroll
        for (int i = 0; i < PER; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, v[i][j] & 0x7fff7fffu));
        return top[0] >= 0x7f80 || top[1] >= 0x7f80;
    }
    __device__ __forceinline__ void drop_not_finite() {
#pragma unroll
        for (int i = 0; i < PER; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t x = v[i][j];
                v[i][j] = ((x & 0x7f800000u) == 0x7f800000u ? 0u : x & 0xffff0000u) | ((x & 0x7f80u) == 0x7f80u ? 0u : x & 0xffffu);
            }
    }
    __device__ __forceinline__ void store(char* tile, int tid) const {
#pragma unroll
        for (int i = 0; i < PER; ++i)
            *reinterpret_cast<u32x4*>(tile + tile_off<DP>(tid / CH + i * (THREADS / CH), tid % CH)) = v[i];
    }
};

// Operands from a tile that begins at a multiple of 256 bytes of LDS, by 32-bit LDS addresses: `at` is the tile's with the lane's part
// (rows_lane, cols_lane) added once, the chunk then an exclusive or and the rows an immediate offset, so that no register holds an address a chunk.
//
// With the contraction along the columns: lane l holds row row0 + l % 32 and columns 16 c + 8 (l / 32) .. + 7; row0 % 32 == 0
typedef __attribute__((address_space(3))) const bf16x8* lds_bf16x8_ptr;
template <int DP>
__device__ __forceinline__ uint32_t rows_lane(int lane) { return tile_off<DP>(lane & 31, lane >> 5); }
template <int DP>
__device__ __forceinline__ bf16x8 frag_rows(uint32_t at, int row0, int c) {
    return *(lds_bf16x8_ptr)(uintptr_t)((at ^ (uint32_t)(c << 5)) + (uint32_t)(row0 * tile_row_bytes<DP>()));
}
// With the contraction along the tokens: lane l holds column 32 db + l % 32 of the tokens row0 + 4 (l / 32) .. + 3 and
// row0 + 8 + 4 (l / 32) .. + 3, the order in which the result of a product lies in registers 8 k .. 8 k + 7; row0 % 16 == 0
template <int DP>
__device__ __forceinline__ uint32_t cols_lane(int lane) {
    return tile_off<DP>(4 * (lane >> 5) + ((lane & 15) >> 2), 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) + (uint32_t)(lane & 1) * 8u;
}
template <int DP>
__device__ __forceinline__ bf16x8 frag_cols(uint32_t at, int row0, int db) {
    const uint32_t lo = (at ^ (uint32_t)(db << 6)) + (uint32_t)(row0 * tile_row_bytes<DP>());
    const uint32_t hi = (at ^ (uint32_t)(db << 6 | 32)) + (uint32_t)((row0 + 8) * tile_row_bytes<DP>());   // 8 rows on: tile_swz differs by 2
    const bf16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_ptr)(uintptr_t)lo);
    const bf16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_ptr)(uintptr_t)hi);
    return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
}
// registers 8 k .. 8 k + 7 of a product, rounded to bf16, as the operand that frag_cols goes with
__device__ __forceinline__ bf16x8 pack_frag(const f32x16& p, int k) {
    u32x4 v;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = pack_bf16x2(p[8 * k + 2 * j], p[8 * k + 2 * j + 1]);
    return __builtin_bit_cast(bf16x8, v);
}
// The same operand from global memory, one row of a head a lane: columns 16 c + 8 (l / 32) .. + 7 of row l % 32
template <int DP>
__device__ __forceinline__ void load_rows(const __amdgpu_buffer_rsrc_t& r, uint32_t row_off, bool ok, int D, int lane, bf16x8 (&f)[DP / 16]) {
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) {
        const int d = 16 * c + 8 * (lane >> 5);
        f[c] = __builtin_bit_cast(bf16x8, buf_load16(r, ok && d < D ? row_off + (uint32_t)d * 2u : kOobOffset));
    }
}

// The same by way of LDS: 32 rows of a wavefront loaded in whole rows (a load of the operand itself touches 32 bytes of each of 32 rows),
// stored to 32 rows of a tile that nobody else uses, and read as operands
template <int DP>
struct RowsIn {
    TileLoad<DP, 32, 64> t;
    __device__ __forceinline__ void load(const bf16_t* base, int stride, int rows, int D, int lane) {
        t.load(HeadRows{base, stride}, 0, rows, D, TileLoad<DP, 32, 64>::first(lane, stride, D));
    }
    __device__ __forceinline__ void operands(char* lds, int lane, bf16x8 (&f)[DP / 16]) const {
        t.store(lds, lane);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const uint32_t at = lds_addr_of(lds) + rows_lane<DP>(lane);
#pragma unroll
        for (int c = 0; c < DP / 16; ++c) f[c] = frag_rows<DP>(at, 0, c);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
};

// What was dropped of a row of values before the products (an infinity or a NaN would make a NaN of a weight of 0), added to the sums of
// those that see it
template <int DP>
__device__ __forceinline__ void add_not_finite(f32x16 (&acc)[DP / 32], const bf16_t* v, int D, int h, bool sees) {
#pragma unroll
    for (int db = 0; db < DP / 32; ++db)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int d = db * 32 + 8 * q + 4 * h;
            const u32x2 x = d < D ? *reinterpret_cast<const u32x2*>(v + d) : u32x2{0, 0};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float f = (e & 1) != 0 ? bf16hi_to_f32(x[e >> 1]) : bf16lo_to_f32(x[e >> 1]);
                acc[db][4 * q + e] += sees && !(fabsf(f) < INFINITY) ? f : 0.0f;
            }
        }
}

// the two halves of a wavefront joined, lane l with lane l + 32
__device__ __forceinline__ float halves_max(float v) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
__device__ __forceinline__ float halves_sum(float v) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}

// The rows of a wavefront from the registers of a product [column][row], lane l columns 32 db + 8 i + 4 (l / 32) .. + 3 of row l % 32, by way of
// LDS (32 rows of a tile that nobody else uses): they leave in whole 256 (128) bytes instead of pieces of 8
template <int DP>
__device__ __forceinline__ void store_rows(bf16_t* base, int stride, int rows, const f32x16 (&acc)[DP / 32], float scale, int D, int lane, char* lds) {
    constexpr int CH = tile_row_bytes<DP>() / 16;
    const int r = lane & 31, h = lane >> 5;
#pragma unroll
    for (int db = 0; db < DP / 32; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const u32x2 w = {pack_bf16x2(acc[db][4 * i] * scale, acc[db][4 * i + 1] * scale),
                             pack_bf16x2(acc[db][4 * i + 2] * scale, acc[db][4 * i + 3] * scale)};
            *reinterpret_cast<u32x2*>(lds + tile_off<DP>(r, db * 4 + i) + 8 * h) = w;
        }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const int c = lane % CH;
#pragma unroll
    for (int i = 0; i < 32 * CH / 64; ++i) {
        const int row = lane / CH + i * (64 / CH);
        const u32x4 v = *reinterpret_cast<const u32x4*>(lds + tile_off<DP>(row, c));
        if (row < rows && c * 8 < D) *reinterpret_cast<u32x4*>(base + (int64_t)row * stride + c * 8) = v;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// ---- which sequence a workgroup works on ---------------------------------------------------------------
// The workgroups of a kernel over packed sequences, the longest first whatever sequence they belong to: the last ones to start are
// the shortest, and the chip empties evenly.  Workgroup j of a sequence has the level top - j num / den (rounded down), in
// 32s of rows that it goes over (num = 0: all the same), so that cnt(L) = ceil((top - L + 1) den / num) of a sequence's have at least L; a search over L finds
// the level of workgroup q, a prefix sum its sequence.  For up to 64 sequences, a lane each; with more of them (each then a small
// part of the whole) workgroups go sequence by sequence.  rows(lengths of a sequence) gives its workgroups and top.
struct SeqItem { int item, q0, q1, k0, k1; };
template <class Rows>
__device__ __forceinline__ bool locate_longest(const AttnArgs& P, int lane, int q, int num, int den, const Rows& rows, SeqItem& it) {
    if (P.n_seq > 64) {
        int cc = 0;
        for (int i0 = 0; i0 < P.n_seq; i0 += 64) {
            int qb = 0, qe = 0, kb = 0, ke = 0, n = 0, top = 0;
            if (i0 + lane < P.n_seq) {
                seg_bounds(P.seg_q, i0 + lane, P.Tq, qb, qe);
                seg_bounds(P.seg_k, i0 + lane, P.Tk, kb, ke);
                rows(qe - qb, ke - kb, n, top);
            }
            const int incl = wave_inclusive_sum(n);
            const uint64_t past = __ballot(q < cc + incl);
            if (past != 0) {
                const int l = __builtin_ctzll(past);
                it = {q - cc - __builtin_amdgcn_readlane(incl - n, l), __builtin_amdgcn_readlane(qb, l), __builtin_amdgcn_readlane(qe, l),
                      __builtin_amdgcn_readlane(kb, l), __builtin_amdgcn_readlane(ke, l)};
                return true;
            }
            cc += __builtin_amdgcn_readlane(incl, 63);
        }
        return false;
    }
    int qb = 0, qe = 0, kb = 0, ke = 0, n = 0, top = 0;
    if (lane < P.n_seq) {
        seg_bounds(P.seg_q, lane, P.Tq, qb, qe);
        seg_bounds(P.seg_k, lane, P.Tk, kb, ke);
        rows(qe - qb, ke - kb, n, top);
    }
    auto at_least = [&](int L) { const int c = top < L ? 0 : num == 0 ? n : ((top - L + 1) * den + num - 1) / num; return c < n ? c : n; };
    int l = 0, item = q, sum = wave_inclusive_sum(n);
    if (q >= __builtin_amdgcn_readlane(sum, 63)) return false;
    if (P.n_seq > 1) {
        // levels of all workgroups lie in (lo, hi]; workgroup q's is the largest L whose workgroups of at least L are more than q
        int hi = n > 0 ? top : -(1 << 30), lo = n > 0 ? top - ((n - 1) * num) / den - 1 : 1 << 30;
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) {
            hi = max(hi, __shfl_xor(hi, off, 64));
            lo = min(lo, __shfl_xor(lo, off, 64));
        }
        hi = __builtin_amdgcn_readfirstlane(hi) + 1;             // none has it
        lo = __builtin_amdgcn_readfirstlane(lo) + 1;             // all have it
        while (hi - lo > 1) {
            const int mid = lo + ((hi - lo) >> 1);
            if (__builtin_amdgcn_readlane(wave_inclusive_sum(at_least(mid)), 63) > q) lo = mid;
            else hi = mid;
        }
        const int before = at_least(lo + 1), here = at_least(lo) - before;
        const int r = q - __builtin_amdgcn_readlane(wave_inclusive_sum(before), 63);
        const int incl = wave_inclusive_sum(here);
        l = __builtin_ctzll(__ballot(r < incl));
        item = r - __builtin_amdgcn_readlane(incl - here, l) + __builtin_amdgcn_readlane(before, l);
    }
    it = {item, __builtin_amdgcn_readlane(qb, l), __builtin_amdgcn_readlane(qe, l), __builtin_amdgcn_readlane(kb, l), __builtin_amdgcn_readlane(ke, l)};
    return true;
}
// workgroup of a kernel by queries: four units of 32 rows of a head, g heads a block of rows, from a sequence's end
__device__ __forceinline__ bool locate_queries(const AttnArgs& P, int lane, int q, int g, SeqItem& it) {
    return locate_longest(P, lane, q, P.causal ? ATT_WAVES : 0, g,
                          [&](int nq, int nk, int& n, int& top) {
                              n = ((nq + ATT_ROWS - 1) / ATT_ROWS * g + ATT_WAVES - 1) / ATT_WAVES;
                              top = (nk + 31) / 32;
                          }, it);
}

// The same value, which the compiler takes for another one: what is computed from it inside a loop is not kept in registers around the loop
__device__ __forceinline__ int unhoisted(int v) {
    asm volatile("" : "+v"(v));
    return v;
}

// A persistent workgroup's k-th piece of `blocks` pieces of work, the longest first: the order is turned round every other time, so
// that who had the longest of one round has the shortest of the next; eight neighbours stay eight neighbours (an XCD each).
__device__ __forceinline__ int piece_of(int k) {
    const int w = (int)blockIdx.x, n = (int)gridDim.x;
    return k * n + ((k & 1) && (n & 7) == 0 ? n - 8 - (w & ~7) + (w & 7) : w);
}

// What a wavefront works on in a kernel by queries: 32 rows of a head
struct QueryUnit {
    int head, row0, wave_end, all_see;                   // keys that the last row, the first row see
    int wg_sees;                                         // keys that every row of the workgroup sees
    int t0, t1;                                          // the workgroup's tiles of keys
    bool any;
};
template <int KEYS>
__device__ __forceinline__ QueryUnit query_unit(const AttnArgs& P, const SeqItem& it, int kvh, int wave, int part = 0, int parts = 1) {
    const int g = P.Hq / P.Hkv, nq = it.q1 - it.q0, nk = it.k1 - it.k0;
    const int units = (nq + ATT_ROWS - 1) / ATT_ROWS * g;
    const int first = units - 1 - it.item * ATT_WAVES, unit = first - wave;       // wave 0 has the latest queries
    auto keys_of = [&](int row) { const int n = P.causal ? row + 1 + nk - nq : nk; return n < nk ? n : nk; };   // may be < 0
    QueryUnit u;
    u.any = unit >= 0;
    u.row0 = u.any ? unit / g * ATT_ROWS : 0;
    u.head = kvh * g + (u.any ? unit % g : 0);
    const int tiles = (max(keys_of(min(first / g * ATT_ROWS + ATT_ROWS, nq) - 1), 0) + KEYS - 1) / KEYS;
    u.t0 = parts == 1 ? 0 : tiles * part / parts;
    u.t1 = parts == 1 ? tiles : tiles * (part + 1) / parts;
    u.wave_end = u.any ? keys_of(min(u.row0 + ATT_ROWS, nq) - 1) : 0;
    u.all_see = keys_of(u.row0);
    u.wg_sees = keys_of(max(first - (ATT_WAVES - 1), 0) / g * ATT_ROWS);
    return u;
}

// Workgroups of a kernel by queries: at least what the sequences take, whatever their lengths (the sum of ceil(ceil(n / 32) g / 4))
inline int64_t attn_query_workgroups(const AttnArgs& a) {
    return (((int64_t)a.Tq / ATT_ROWS + a.n_seq) * (a.Hq / a.Hkv) / ATT_WAVES + a.n_seq) * a.Hkv;
}

}  // namespace skipffn
