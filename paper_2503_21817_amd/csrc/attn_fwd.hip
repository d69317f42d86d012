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

// Workgroups that fit a compute unit at a time
template <int DP> constexpr int fwd_per_cu() { return DP <= 64 ? 3 : 2; }

template <int DP>
__global__ __launch_bounds__(ATT_THREADS, fwd_per_cu<DP>()) void attn_fwd_kernel(const AttnArgs P, const int blocks) {
    constexpr int TILE = FWD_KEYS * tile_row_bytes<DP>();
    __shared__ __align__(256) char smem[4 * TILE];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5;
    const int g = P.Hq / P.Hkv;
    int kvh, turn = 0;
    SeqItem it;
    auto locate = [&](int k, int& head, SeqItem& to) {
        const int piece = piece_of(k);
        if (piece >= blocks) return false;
        head = piece % P.Hkv;
        return locate_queries(P, unhoisted(lane), piece / P.Hkv, g, to);
    };
    const uint32_t k_off = TileLoad<DP, FWD_KEYS>::first(tid, P.k_tok, P.D), v_off = TileLoad<DP, FWD_KEYS>::first(tid, P.v_tok, P.D);
    const uint32_t rows_at = lds_addr_of(smem) + rows_lane<DP>(lane), cols_at = lds_addr_of(smem) + TILE + cols_lane<DP>(lane);
    TileLoad<DP, FWD_KEYS> lk, lv;
    auto load_tile = [&](const SeqItem& s, int head, int t) {
        lk.load(HeadRows{P.k + head * P.k_head + (int64_t)s.k0 * P.k_tok, P.k_tok}, t * FWD_KEYS, s.k1 - s.k0, P.D, k_off);
        lv.load(HeadRows{P.v + head * P.v_head + (int64_t)s.k0 * P.v_tok, P.v_tok}, t * FWD_KEYS, s.k1 - s.k0, P.D, v_off);
    };
    bf16x8 qf[DP / 16];
    auto load_q = [&](const SeqItem& s, const QueryUnit& u) {
        const int ln = unhoisted(lane);
        load_rows<DP>(make_rsrc(P.q + u.head * P.q_head + (int64_t)(s.q0 + u.row0) * P.q_tok, 0x7fffffffu), (uint32_t)((ln & 31) * P.q_tok) * 2u,
                      u.any && u.row0 + (ln & 31) < s.q1 - s.q0, P.D, ln, qf);
    };
    if (!locate(0, kvh, it)) return;
    QueryUnit u = query_unit<FWD_KEYS>(P, it, kvh, wave);
    load_q(it, u);
    if (u.tiles > 0) load_tile(it, kvh, 0);
    int stage = 0;                                       // which of the two tiles in LDS
    for (;;) {
        SeqItem next_it;
        int next_kvh = 0;
        const bool more = locate(++turn, next_kvh, next_it);
        const QueryUnit next = more ? query_unit<FWD_KEYS>(P, next_it, next_kvh, wave) : QueryUnit{};
        const int nq = it.q1 - it.q0, nk = it.k1 - it.k0, row = u.row0 + (lane & 31);
        const int row_keys = P.causal ? min(row + 1 + nk - nq, nk) : nk;
        f32x16 acc[DP / 32] = {};
        float m = -INFINITY, l = 0.0f;
        const float c = P.scale_log2;
        if (u.tiles > 0) {
            lk.store(smem + stage * 2 * TILE, tid);
            lv.store(smem + stage * 2 * TILE + TILE, tid);
            __syncthreads();
        } else if (next.tiles > 0) {
            load_tile(next_it, next_kvh, 0);
        }
        for (int t = 0; t < u.tiles; ++t) {
            const uint32_t at = (uint32_t)stage * (2 * TILE), tk = rows_at + at, tv = cols_at + at;
            const bool last = t + 1 == u.tiles;
            if (!last) load_tile(it, kvh, t + 1);
            else if (next.tiles > 0) load_tile(next_it, next_kvh, 0);
            if (t * FWD_KEYS < u.wave_end) {
                f32x16 s[2];
                __builtin_amdgcn_s_setprio(1);
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) {
                    s[kb] = f32x16{};
#pragma unroll
                    for (int d = 0; d < DP / 16; ++d)
                        s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_rows<DP>(tk, kb * 32, d), qf[d], s[kb], 0, 0, 0);
                }
                __builtin_amdgcn_s_setprio(0);
                if ((t + 1) * FWD_KEYS > u.all_see) {
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
            if (!last) {
                stage ^= 1;
                lk.store(smem + stage * 2 * TILE, tid);
                lv.store(smem + stage * 2 * TILE + TILE, tid);
                __syncthreads();
            }
        }
        if (more) load_q(next_it, next);
        l = halves_sum(l);
        if (u.any) {
            const float inv = l == 0.0f ? 0.0f : 1.0f / l;   // a row that sees no key is zero
            // by way of the tile that no wavefront reads any more
            store_rows<DP>(P.out + u.head * P.o_head + (int64_t)(it.q0 + u.row0) * P.o_tok, P.o_tok, min(nq - u.row0, ATT_ROWS), acc, inv, P.D,
                           unhoisted(lane), smem + (stage ^ 1) * 2 * TILE + wave * 32 * tile_row_bytes<DP>());
            if (P.lse != nullptr && h == 0 && row < nq)
                P.lse[(int64_t)u.head * P.Tq + it.q0 + row] = l == 0.0f ? INFINITY : fmaf(m, c, __builtin_amdgcn_logf(l));
        }
        if (!more) return;
        __syncthreads();                                 // both tiles have been read
        it = next_it;
        kvh = next_kvh;
        u = next;
    }
}

hipError_t launch_attn_forward(const AttnArgs& a, int ncu, hipStream_t s) {
    const int64_t blocks = attn_query_workgroups(a);
    const int64_t fit = (int64_t)ncu * (a.D <= 64 ? fwd_per_cu<64>() : fwd_per_cu<128>()) / 8 * 8;
    const dim3 grid((uint32_t)(blocks < fit ? blocks : fit));
    if (a.D <= 64) attn_fwd_kernel<64><<<grid, ATT_THREADS, 0, s>>>(a, (int)blocks);
    else attn_fwd_kernel<128><<<grid, ATT_THREADS, 0, s>>>(a, (int)blocks);
    return hipGetLastError();
}

}  // namespace skipffn
