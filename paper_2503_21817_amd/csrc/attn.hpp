// Attention of packed sequences on v_mfma_f32_32x32x16_bf16: what the forward, the backward and the single-token kernels share.
//
// With S = scale Q K^T over the keys a row sees, P = softmax(S) by rows and O = P V.  Every product is taken with the result
// transposed so that the exponentials a lane computes are already an operand of the next product:
//   S^T [key][query] = K Q^T    leaves a lane one query (column lane % 32) and 16 of 32 keys (8 (i / 4) + 4 (lane / 32) + i % 4);
//   O^T [d][query] = V^T P^T    takes the same registers, rounded to bf16, as its second operand: the order of the contraction is
//                               free, so V^T is read in the order of keys that the lane holds.
// Row maxima and sums then stay inside a lane but for one exchange with the lane 32 further.
//
// A tile of rows [token][column] of one head lies in LDS with 256 (128) bytes a row for heads of up to 128 (64) columns, 16-byte
// chunk c of row r at c ^ tile_swz(r).  The same placing serves both ways it is read, free of bank conflicts: 16 consecutive rows
// at one chunk (ds_read_b128, the operand whose contraction runs along the columns) and 4 rows x 64 bytes (ds_read_b64_tr_b16, the
// operand whose contraction runs along the tokens).
#pragma once

#include "kernels.hpp"
#include "segments.hpp"

namespace skipffn {

constexpr int ATT_ROWS = 32;               // queries of a wavefront
constexpr int ATT_WAVES = 4;
constexpr int ATT_THREADS = ATT_WAVES * 64;
constexpr float kLog2e = 1.4426950408889634f;

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

// A tile of N rows on its way through registers: issued as buffer loads, stored to LDS a tile later.  Rows at and past `rows`
// and columns at and past the head's read zeros (so a masked weight of 0 never meets what lies there).
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
    __device__ __forceinline__ void store(char* tile, int tid) const {
#pragma unroll
        for (int i = 0; i < PER; ++i)
            *reinterpret_cast<u32x4*>(tile + tile_off<DP>(tid / CH + i * (THREADS / CH), tid % CH)) = v[i];
    }
};

// Operand with the contraction along the columns: lane l holds row row0 + l % 32 and columns 16 c + 8 (l / 32) .. + 7
template <int DP>
__device__ __forceinline__ bf16x8 frag_rows(const char* tile, int row0, int c, int lane) {
    return *reinterpret_cast<const bf16x8*>(tile + tile_off<DP>(row0 + (lane & 31), 2 * c + (lane >> 5)));
}
// Operand with the contraction along the tokens: lane l holds column 32 db + l % 32 of the tokens row0 + 4 (l / 32) .. + 3 and
// row0 + 8 + 4 (l / 32) .. + 3, the order in which the result of a product lies in registers 8 k .. 8 k + 7
template <int DP>
__device__ __forceinline__ bf16x8 frag_cols(char* tile, int row0, int db, int lane) {
    const int r = row0 + 4 * (lane >> 5) + ((lane & 15) >> 2);
    const int chunk = 4 * db + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), half = (lane & 1) * 8;
    const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_ptr)(tile + tile_off<DP>(r, chunk) + half));
    const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_ptr)(tile + tile_off<DP>(r + 8, chunk) + half));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
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

// the two halves of a wavefront joined, lane l with lane l + 32
__device__ __forceinline__ float halves_max(float v) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
__device__ __forceinline__ float halves_sum(float v) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}

// A row of the result from the registers of a product [column][row]: lane l has the row l % 32 and columns 32 db + 8 i + 4 (l / 32) .. + 3
template <int DP>
__device__ __forceinline__ void store_cols(bf16_t* row, const f32x16 (&acc)[DP / 32], float scale, int D, int h) {
#pragma unroll
    for (int db = 0; db < DP / 32; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int d = db * 32 + 8 * i + 4 * h;
            if (d < D) {
                const u32x2 w = {pack_bf16x2(acc[db][4 * i] * scale, acc[db][4 * i + 1] * scale),
                                 pack_bf16x2(acc[db][4 * i + 2] * scale, acc[db][4 * i + 3] * scale)};
                *reinterpret_cast<u32x2*>(row + d) = w;
            }
        }
}

// ---- which sequence a workgroup works on ---------------------------------------------------------------
// Set s has items(its length) workgroups; workgroup q of all -> s, its index among the set's, and the set's bounds, which
// bounds(s, b, e) gives.  False past the last one.  A lane takes a set, a prefix sum over the lanes finds the workgroup's (whole
// wavefronts).
template <class Bounds, class Items>
__device__ __forceinline__ bool locate_in(int S, int q, const Bounds& bounds, const Items& items, int& s, int& item, int& t0, int& t1) {
    const int lane = threadIdx.x & 63;
    int cc = 0;
    for (int i0 = 0; i0 < S; i0 += 64) {
        int b = 0, e = 0;
        if (i0 + lane < S) bounds(i0 + lane, b, e);
        const int nc = items(e - b);
        const int incl = wave_inclusive_sum(nc);
        const uint64_t past = __ballot(q < cc + incl);
        if (past != 0) {
            const int l = __builtin_ctzll(past);
            t0 = __builtin_amdgcn_readlane(b, l);
            t1 = __builtin_amdgcn_readlane(e, l);
            s = i0 + l;
            item = q - cc - __builtin_amdgcn_readlane(incl - nc, l);
            return true;
        }
        cc += __builtin_amdgcn_readlane(incl, 63);
    }
    return false;
}
template <class Items>
__device__ __forceinline__ bool locate_item(const int32_t* __restrict__ seg, int S, int n_tok, int q, const Items& items,
                                            int& s, int& item, int& t0, int& t1) {
    return locate_in(S, q, [&](int i, int& b, int& e) { seg_bounds(seg, i, n_tok, b, e); }, items, s, item, t0, t1);
}

// Workgroups of a kernel by queries: at least what the sequences take, whatever their lengths (the sum of ceil(ceil(n / 32) g / 4))
inline int64_t attn_query_workgroups(const AttnArgs& a) {
    return (((int64_t)a.Tq / ATT_ROWS + a.n_seq) * (a.Hq / a.Hkv) / ATT_WAVES + a.n_seq) * a.Hkv;
}

}  // namespace skipffn
