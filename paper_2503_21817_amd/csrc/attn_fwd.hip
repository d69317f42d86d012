// Attention over whole prompts, forward: out_i = sum_j softmax_j(scale q_i . k_j) v_j over the keys j that row i sees.
//
// One pass over the keys with the running maximum and sum of the softmax.  A workgroup of four wavefronts works on four units - a
// unit is 32 consecutive queries of a sequence in one head - of the same sequence and key/value head, the heads of a group first,
// and takes tiles of 64 keys and values through LDS, two tiles deep: the next tile's loads are under way in registers while this
// one is worked on.  With 8 heads a chip-wide row of 8 workgroups has one key/value head each, so that an XCD's L2 holds one
// head's keys.  Units of a sequence are taken from its end: in a causal prompt the longest first.
#include "attn.hpp"

namespace skipffn {

constexpr int FWD_KEYS = 64;

template <int DP>
__global__ __launch_bounds__(ATT_THREADS, 2) void attn_fwd_kernel(const AttnArgs P) {
    constexpr int TILE = FWD_KEYS * tile_row_bytes<DP>();
    __shared__ __align__(256) char smem[4 * TILE];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5;
    const int kvh = (int)blockIdx.x % P.Hkv, g = P.Hq / P.Hkv;
    SeqItem it;
    if (!locate_queries(P, (int)blockIdx.x / P.Hkv, g, it)) return;
    const int item = it.item, q0 = it.q0, q1 = it.q1, k0 = it.k0, k1 = it.k1;
    const int nq = q1 - q0, nk = k1 - k0, ahead = nk - nq;
    const int units = (nq + ATT_ROWS - 1) / ATT_ROWS * g;
    const int first = units - 1 - item * ATT_WAVES, unit = first - wave;          // wave 0 has the latest queries
    const int row0 = unit >= 0 ? unit / g * ATT_ROWS : 0, head = kvh * g + (unit >= 0 ? unit % g : 0);
    auto keys_of = [&](int row) { const int n = P.causal ? row + 1 + ahead : nk; return n < nk ? n : nk; };   // of a query; may be < 0
    const int last = first / g * ATT_ROWS + ATT_ROWS;
    const int tiles = (max(keys_of((last < nq ? last : nq) - 1), 0) + FWD_KEYS - 1) / FWD_KEYS;
    const int wave_end = unit >= 0 ? keys_of((row0 + ATT_ROWS < nq ? row0 + ATT_ROWS : nq) - 1) : 0;
    const int all_see = keys_of(row0);                                           // keys before it are seen by every row

    const int row = row0 + (lane & 31);
    const bool row_ok = unit >= 0 && row < nq;
    const int row_keys = keys_of(row);
    bf16x8 qf[DP / 16];
    {
        const __amdgpu_buffer_rsrc_t rq = make_rsrc(P.q + head * P.q_head + (int64_t)(q0 + row0) * P.q_tok, 0x7fffffffu);
        load_rows<DP>(rq, (uint32_t)((lane & 31) * P.q_tok) * 2u, row_ok, P.D, lane, qf);
    }
    const HeadRows K{P.k + kvh * P.k_head + (int64_t)k0 * P.k_tok, P.k_tok}, V{P.v + kvh * P.v_head + (int64_t)k0 * P.v_tok, P.v_tok};
    const uint32_t k_off = TileLoad<DP, FWD_KEYS>::first(tid, P.k_tok, P.D), v_off = TileLoad<DP, FWD_KEYS>::first(tid, P.v_tok, P.D);
    TileLoad<DP, FWD_KEYS> lk, lv;
    const uint32_t rows_at = lds_addr_of(smem) + rows_lane<DP>(lane), cols_at = lds_addr_of(smem) + TILE + cols_lane<DP>(lane);

    f32x16 acc[DP / 32] = {};
    float m = -INFINITY, l = 0.0f;
    const float c = P.scale_log2;
    if (tiles > 0) {
        lk.load(K, 0, nk, P.D, k_off);
        lv.load(V, 0, nk, P.D, v_off);
        lk.store(smem, tid);
        lv.store(smem + TILE, tid);
    }
    __syncthreads();
    for (int t = 0; t < tiles; ++t) {
        const uint32_t stage = (uint32_t)(t & 1) * (2 * TILE), tk = rows_at + stage, tv = cols_at + stage;
        if (t + 1 < tiles) {
            lk.load(K, (t + 1) * FWD_KEYS, nk, P.D, k_off);
            lv.load(V, (t + 1) * FWD_KEYS, nk, P.D, v_off);
        }
        if (t * FWD_KEYS < wave_end) {
            f32x16 s[2];
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                s[kb] = f32x16{};
#pragma unroll
                for (int d = 0; d < DP / 16; ++d)
                    s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_rows<DP>(tk, kb * 32, d), qf[d], s[kb], 0, 0, 0);
            }
            if ((t + 1) * FWD_KEYS > all_see) {
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (t * FWD_KEYS + kb * 32 + 8 * (i >> 2) + 4 * h + (i & 3) >= row_keys) s[kb][i] = -INFINITY;
            }
            float top = s[0][0];
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i) top = fmaxf(top, s[kb][i]);
            top = halves_max(top);
            // The maximum may lag by up to a factor 2^8 of the weights, which bf16 and the fp32 sums hold as exactly: the sums are
            // seldom scaled again
            if (__ballot((top - m) * c > 8.0f || (m == -INFINITY && top != -INFINITY)) != 0) {
                const float now = fmaxf(m, top), scale = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - now) * c);
                l *= scale;
#pragma unroll
                for (int db = 0; db < DP / 32; ++db)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[db][i] *= scale;
                m = now;
            }
            const float mc = m == -INFINITY ? 0.0f : m * c;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    s[kb][i] = __builtin_amdgcn_exp2f(fmaf(s[kb][i], c, -mc));
                    l += s[kb][i];
                }
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const bf16x8 p = pack_frag(s[kb], k);
#pragma unroll
                    for (int db = 0; db < DP / 32; ++db)
                        acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_cols<DP>(tv, kb * 32 + k * 16, db), p, acc[db], 0, 0, 0);
                }
        }
        if (t + 1 < tiles) {
            char* nx = smem + ((t + 1) & 1) * 2 * TILE;
            lk.store(nx, tid);
            lv.store(nx + TILE, tid);
        }
        __syncthreads();
    }
    l = halves_sum(l);
    if (unit < 0) return;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;          // a row that sees no key is zero
    store_rows<DP>(P.out + head * P.o_head + (int64_t)(q0 + row0) * P.o_tok, P.o_tok, min(nq - row0, ATT_ROWS), acc, inv, P.D, lane,
                   smem + wave * 32 * tile_row_bytes<DP>());
    if (P.lse != nullptr && h == 0 && row_ok)
        P.lse[(int64_t)head * P.Tq + q0 + row] = l == 0.0f ? INFINITY : fmaf(m, c, __builtin_amdgcn_logf(l));
}

hipError_t launch_attn_forward(const AttnArgs& a, hipStream_t s) {
    const dim3 grid((uint32_t)attn_query_workgroups(a));
    if (a.D <= 64) attn_fwd_kernel<64><<<grid, ATT_THREADS, 0, s>>>(a);
    else attn_fwd_kernel<128><<<grid, ATT_THREADS, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace skipffn
