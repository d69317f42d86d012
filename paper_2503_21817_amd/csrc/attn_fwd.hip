// Attention over whole prompts, forward: out_i = sum_j softmax_j(scale q_i . k_j) v_j over the keys j that row i sees.
//
// One pass over the keys with the running maximum and sum of the softmax.  A workgroup of four wavefronts works on four units - a
// unit is 32 consecutive queries of a sequence in one head - of the same sequence and key/value head, the heads of a group first,
// and takes tiles of 64 or 32 keys and values through LDS, two tiles deep: the next tile's loads are under way in registers while this
// one is worked on.  With 8 heads a chip-wide row of 8 workgroups has one key/value head each, so that an XCD's L2 holds one
// head's keys.  Units of a sequence are taken from its end: in a causal prompt the longest first.
//
// Long prompts are bound by the power limit (the chip falls to 1.42-1.85 GHz, by the card, with the matrix cores busy 50-56 % of the time): 1 x 16384 tokens,
// 32 / 8 heads of 128, 2030-2325 us by the card, 945-1083 TFLOP/s of what the mask leaves, a library product of 8192^3 reaching 1150-1190.  Short ones
// by the bytes of q and out, which a workgroup's products do not hide: 8 x 616 tokens 48 us, 520 TFLOP/s and 2.1 TB/s.
#include "attn.hpp"

namespace skipffn {

// Workgroups a compute unit and keys a tile.  With pieces for all of them three workgroups (168 registers) do better than two, as some load
// or store while others work; at 128 columns that leaves room for tiles of 32 keys.  64 keys and two workgroups / 32 and three, us:
// 16 x 616 tokens 94 / 89, 32 x 200 45.8 / 40, 16 x up to 3080 729 / 711, 4 x 4096 605 / 608, 1 x 16384 2271 / 2275 (the power limit); but with fewer pieces than two a unit,
// where a workgroup has its SIMDs to itself: 4 x 47 after 640 17.1 / 19.1.  64 columns, 64 keys and three / 32 and four: 8 x 577 25.4 / 26.6.
template <int DP, int KEYS> constexpr int fwd_per_cu() { return DP <= 64 || KEYS == 32 ? 3 : 2; }

template <int DP, int KEYS, bool PARTS>
__global__ __launch_bounds__(ATT_THREADS, (fwd_per_cu<DP, KEYS>())) void attn_fwd_kernel(const AttnArgs P, const int blocks) {
    constexpr int KB = KEYS / 32, TILE = KEYS * tile_row_bytes<DP>(), ROWS = ATT_WAVES * 32 * tile_row_bytes<DP>();
    __shared__ __align__(256) char smem[4 * TILE];
    __shared__ int dropped_in[ATT_WAVES];                // by wavefront: the last piece in whose tiles it dropped a value
    static_assert(4 * TILE >= ROWS, "the rows of a piece leave by way of the tiles");
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5;
    const int g = P.Hq / P.Hkv;
    int kvh, turn = 0, part = 0;                         // part: of the keys
    SeqItem it;
    auto locate = [&](int k, int& head, int& z, SeqItem& to) {
        int piece = piece_of(k);
        if (piece >= blocks) return false;
        head = piece % P.Hkv;
        piece /= P.Hkv;
        if constexpr (PARTS) {
            z = piece % P.splits;
            piece /= P.splits;
        }
        return locate_queries(P, unhoisted(lane), piece, g, to);
    };
    const uint32_t k_off = TileLoad<DP, KEYS>::first(tid, P.k_tok, P.D), v_off = TileLoad<DP, KEYS>::first(tid, P.v_tok, P.D);
    const uint32_t rows_at = lds_addr_of(smem) + rows_lane<DP>(lane), cols_at = lds_addr_of(smem) + TILE + cols_lane<DP>(lane);
    TileLoad<DP, KEYS> lk, lv;
    auto load_tile = [&](const SeqItem& s, int head, int t) {
        lk.load(HeadRows{P.k + head * P.k_head + (int64_t)s.k0 * P.k_tok, P.k_tok}, t * KEYS, s.k1 - s.k0, P.D, k_off);
        lv.load(HeadRows{P.v + head * P.v_head + (int64_t)s.k0 * P.v_tok, P.v_tok}, t * KEYS, s.k1 - s.k0, P.D, v_off);
    };
    bf16x8 qf[DP / 16];
    auto load_q = [&](const SeqItem& s, const QueryUnit& u) {
        const int ln = unhoisted(lane);
        load_rows<DP>(make_rsrc(P.q + u.head * P.q_head + (int64_t)(s.q0 + u.row0) * P.q_tok, 0x7fffffffu), (uint32_t)((ln & 31) * P.q_tok) * 2u,
                      u.any && u.row0 + (ln & 31) < s.q1 - s.q0, P.D, ln, qf);
    };
    if (!locate(0, kvh, part, it)) return;
    if (lane == 0) dropped_in[wave] = 0;
    QueryUnit u = query_unit<KEYS>(P, it, kvh, wave, part, PARTS ? P.splits : 1);
    load_q(it, u);
    if (u.t0 < u.t1) load_tile(it, kvh, u.t0);
    int stage = 0;                                       // which of the two tiles in LDS
    for (;;) {
        SeqItem next_it;
        int next_kvh = 0, next_part = 0;
        const bool more = locate(++turn, next_kvh, next_part, next_it);
        const QueryUnit next = more ? query_unit<KEYS>(P, next_it, next_kvh, wave, next_part, PARTS ? P.splits : 1) : QueryUnit{};
        const int nq = it.q1 - it.q0, nk = it.k1 - it.k0, row = u.row0 + (lane & 31);
        const int row_keys = P.causal ? min(row + 1 + nk - nq, nk) : nk;
        f32x16 acc[DP / 32] = {};
        float m = -INFINITY, l = 0.0f;
        const float c = P.scale_log2;
        // a tile of which a row does not see every key: values that are not finite leave it, and are added at the end
        auto store_tile = [&](int t) {
            if (P.causal && (t + 1) * KEYS > u.wg_sees && lv.any_not_finite()) {
                lv.drop_not_finite();
                dropped_in[wave] = turn;
            }
            lk.store(smem + stage * 2 * TILE, tid);
            lv.store(smem + stage * 2 * TILE + TILE, tid);
            __syncthreads();
        };
        if (u.t0 < u.t1) {
            store_tile(u.t0);
        } else if (next.t0 < next.t1) {
            load_tile(next_it, next_kvh, next.t0);
        }
        auto work_on = [&](int t) {
            if (t * KEYS >= u.wave_end) return;
            const uint32_t at = (uint32_t)stage * (2 * TILE), tk = rows_at + at, tv = cols_at + at;
            // Operands are asked for a few products ahead and the order is held (left to itself the compiler reads each right before its
            // product); products go before the other wavefront's exponentials.  1 x 16384 tokens 2127 -> 2030 us, 1 x 616 21.7 -> 17.8
            f32x16 s[KB];
            constexpr int NK = DP / 16, AHEAD = KB + 2;
            {
                bf16x8 kf[AHEAD];
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) kf[i] = frag_rows<DP>(tk, i / NK * 32, i % NK);
                __builtin_amdgcn_s_setprio(1);
#pragma unroll
                for (int i = 0; i < KB * NK; ++i) {
                    __builtin_amdgcn_sched_barrier(0);
                    if (i % NK == 0) s[i / NK] = f32x16{};
                    s[i / NK] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[i % AHEAD], qf[i % NK], s[i / NK], 0, 0, 0);
                    if (i + AHEAD < KB * NK) kf[i % AHEAD] = frag_rows<DP>(tk, (i + AHEAD) / NK * 32, (i + AHEAD) % NK);
                }
                __builtin_amdgcn_sched_barrier(0);
                __builtin_amdgcn_s_setprio(0);
            }
            if ((t + 1) * KEYS > u.all_see) {
#pragma unroll
                for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (t * KEYS + kb * 32 + 8 * (i >> 2) + 4 * h + (i & 3) >= row_keys) s[kb][i] = -INFINITY;
            }
            float top = s[0][0];
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i) top = fmaxf(top, s[kb][i]);
            top = halves_max(top);
            // The maximum may lag by up to a factor 2^8 of the weights, which bf16 and the fp32 sums hold as exactly: the sums are
            // seldom scaled again.  Each row by its own scores: what its neighbours in the product see does not change how its weights are rounded
            const bool grow = (top - m) * c > 8.0f || (m == -INFINITY && top != -INFINITY);
            if (__ballot(grow) != 0) {
                const float now = grow ? fmaxf(m, top) : m, scale = grow ? __builtin_amdgcn_exp2f((m - now) * c) : 1.0f;
                l *= scale;
#pragma unroll
                for (int db = 0; db < DP / 32; ++db)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[db][i] *= scale;
                m = now;
            }
            const float mc = m == -INFINITY ? 0.0f : m * c;
            auto weight = [&](int kb, int i) {
                s[kb][i] = __builtin_amdgcn_exp2f(fmaf(s[kb][i], c, -mc));
                l += s[kb][i];
            };
            constexpr int NV = DP / 32, VAHEAD = KB + 1, STEPS = 2 * KB * NV;
            bf16x8 vf[VAHEAD], pf;
#pragma unroll
            for (int i = 0; i < VAHEAD; ++i) vf[i] = frag_cols<DP>(tv, i / NV * 16, i % NV);
#pragma unroll
            for (int i = 0; i < 8; ++i) weight(0, i);    // of the first product's keys; the others beside the products
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                __builtin_amdgcn_sched_barrier(0);
                if (i % NV == 0) pf = pack_frag(s[i / NV >> 1], i / NV & 1);
                acc[i % NV] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[i % VAHEAD], pf, acc[i % NV], 0, 0, 0);
                if (i + VAHEAD < STEPS) vf[i % VAHEAD] = frag_cols<DP>(tv, (i + VAHEAD) / NV * 16, (i + VAHEAD) % NV);
                if (i < (2 * KB - 1) * NV) {
#pragma unroll
                    for (int w = 8 + i * 8 / NV; w < 8 + (i + 1) * 8 / NV; ++w) weight(w >> 4, w & 15);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(0);
        };
        for (int t = u.t0; t + 1 < u.t1; ++t) {
            load_tile(it, kvh, t + 1);
            work_on(t);
            stage ^= 1;
            store_tile(t + 1);
        }
        if (u.t0 < u.t1) {
            if (next.t0 < next.t1) load_tile(next_it, next_kvh, next.t0);
            work_on(u.t1 - 1);
        }
        bool dropped = false;
#pragma unroll
        for (int i = 0; i < ATT_WAVES; ++i) dropped |= dropped_in[i] == turn;
        if (P.causal && __ballot(dropped) != 0) {
            const int end = min(u.t1 * KEYS, u.wave_end);
            for (int j = max(u.t0, max(u.wg_sees, 0) / KEYS) * KEYS; j < end; ++j)
                add_not_finite<DP>(acc, P.v + kvh * P.v_head + (int64_t)(it.k0 + j) * P.v_tok, P.D, h, j < row_keys);
        }
        if constexpr (2 * TILE < ROWS) __syncthreads();  // otherwise the rows fit the tile that no wavefront reads any more
        if (more) load_q(next_it, next);
        l = halves_sum(l);
        if (PARTS && u.any) {
            // keys seen, all with scores of minus infinity: not the infinity of a part without any (see attn_join.hip)
            if (u.t0 < u.t1 && row_keys > u.t0 * KEYS) m = fmaxf(m, -FLT_MAX);
            if (row < nq) {
                const int64_t at = ((int64_t)(it.q0 + row) * P.Hq + u.head) * P.splits + part;
                if (h == 0) {
                    P.stat[2 * at] = m;
                    P.stat[2 * at + 1] = l;
                }
#pragma unroll
                for (int db = 0; db < DP / 32; ++db)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        *reinterpret_cast<f32x4*>(P.part + at * attn_padded_columns(DP) + db * 32 + 8 * i + 4 * h) =
                            f32x4{acc[db][4 * i], acc[db][4 * i + 1], acc[db][4 * i + 2], acc[db][4 * i + 3]};
            }
        } else if (u.any) {
            // A row that sees no key is zero.  One that does has a weight of 1 at its maximum; if all its scores are minus infinity it is 0 / 0
            const bool none = row_keys <= 0;
            const float inv = none ? 0.0f : 1.0f / l;
            store_rows<DP>(P.out + u.head * P.o_head + (int64_t)(it.q0 + u.row0) * P.o_tok, P.o_tok, min(nq - u.row0, ATT_ROWS), acc, inv, P.D,
                           unhoisted(lane), smem + (2 * TILE < ROWS ? 0 : (stage ^ 1) * 2 * TILE) + wave * 32 * tile_row_bytes<DP>());
            if (P.lse != nullptr && h == 0 && row < nq)
                P.lse[(int64_t)u.head * P.Tq + it.q0 + row] = none ? INFINITY : fmaf(m, c, __builtin_amdgcn_logf(l));
        }
        if (!more) return;
        __syncthreads();                                 // both tiles have been read
        it = next_it;
        kvh = next_kvh;
        part = next_part;
        u = next;
    }
}

// Few queries over many keys would leave most of the chip idle.  The lengths are on the device: this goes by the average number of keys a sequence.  Parts cost a second kernel (about 4 us) and a row of fp32 written
// and read again each (at about 4 TB/s), and save tiles of keys one after the other (about 1.2 us each)
int attn_forward_splits(int64_t Tq, int64_t Tk, int64_t n_seq, int64_t Hq, int64_t Hkv, int64_t D, int ncu) {
    if (Tq <= 0 || Tk <= 0 || n_seq <= 0) return 1;
    AttnArgs a{};
    a.Tq = (int)Tq; a.n_seq = (int)n_seq; a.Hq = (int)Hq; a.Hkv = (int)Hkv;
    const int64_t blocks = attn_query_workgroups(a), fit = (int64_t)ncu * 2;
    const double tiles = (double)Tk / (double)n_seq / 64.0, row_us = (double)Tq * (double)Hq * (attn_padded_columns((int)D) * 8) / 4e6;
    int best = 1;
    double least = tiles * 1.2;
    for (int n = 2; n <= 16 && n <= tiles && blocks * n <= fit; ++n) {
        const double us = tiles * 1.2 / n + 4.0 + row_us * n;
        if (us < least) { least = us; best = n; }
    }
    return best;
}

template <int DP, int KEYS, bool PARTS>
static void launch_fwd(const AttnArgs& a, int64_t blocks, int ncu, hipStream_t s) {
    const int64_t fit = (int64_t)ncu * fwd_per_cu<DP, KEYS>() / 8 * 8;
    attn_fwd_kernel<DP, KEYS, PARTS><<<dim3((uint32_t)(blocks < fit ? blocks : fit)), ATT_THREADS, 0, s>>>(a, (int)blocks);
}

hipError_t launch_attn_forward(const AttnArgs& a, int ncu, hipStream_t s) {
    const int64_t blocks = attn_query_workgroups(a) * a.splits;
    if (a.D <= 64 && a.splits > 1) launch_fwd<64, 64, true>(a, blocks, ncu, s);
    else if (a.D <= 64) launch_fwd<64, 64, false>(a, blocks, ncu, s);
    else if (a.splits > 1 && a.D <= 96) launch_fwd<96, 64, true>(a, blocks, ncu, s);
    else if (a.splits > 1) launch_fwd<128, 64, true>(a, blocks, ncu, s);
    else if (blocks <= 2 * ncu && a.D <= 96) launch_fwd<96, 64, false>(a, blocks, ncu, s);
    else if (blocks <= 2 * ncu) launch_fwd<128, 64, false>(a, blocks, ncu, s);
    else if (a.D <= 96) launch_fwd<96, 32, false>(a, blocks, ncu, s);
    else launch_fwd<128, 32, false>(a, blocks, ncu, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    AttnJoinArgs j{};
    j.T = a.Tq; j.Hq = a.Hq; j.D = a.D; j.splits = a.splits; j.scale_log2 = a.scale_log2;
    j.part = a.part; j.stat = a.stat;
    j.out = a.out; j.o_tok = a.o_tok; j.o_head = a.o_head;
    j.lse = a.lse;
    j.seg = a.seg_q; j.n_seq = a.n_seq;
    return launch_attn_join(j, s);
}

}  // namespace skipffn
