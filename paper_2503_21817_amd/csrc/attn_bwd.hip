// Attention over whole prompts, backward.  With P_ij = exp(S_ij - lse_i), S = scale Q K^T, and delta_i = dO_i . o_i
// (= sum_j P_ij dP_ij, as o is the normalised output):
//     dP = dO V^T,  dS = P (dP - delta),  dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO
// with dK and dV summed over the query heads of a key/value head.  P is computed again from the saved log-sum-exp, so nothing of
// size queries x keys is kept.  Two kernels, each the owner of what it writes, so that no sum depends on an order of atomics:
// one by queries (dQ, and delta on the way), one by keys (dK, dV).  That is 7 products for the 5 that one kernel would take, and
// no fp32 traffic for partial dQ.  The weights and dS are rounded to bf16 for the products they enter, as the matrix cores want them; delta
// and everything summed is fp32.
//
// dQ is bound by power in long prompts, dK and dV less so (matrix cores busy 49 % of the time at the clock at which dQ has 56 %: their causal pieces are up to
// a third longer than an even share); both by the bytes of q, out and their gradients in short ones.  32 / 8 heads of 128, us (TFLOP/s of each kernel's own
// products), by the card: 4 x 2944 tokens dQ 410-456 (935-1040), dK and dV 637-705 (805-890); 16 x 616 dQ 125-138 (540-600), dK and dV 156-174 (570-640).
#include <algorithm>

#include "attn.hpp"

namespace skipffn {

constexpr int DQ_KEYS = 64;

// ---- dQ, delta: a wavefront has a unit of 32 queries of one head, as in the forward kernel ------------------------------------
// Two workgroups a compute unit: the queries and their gradients stay in registers (64 of them) beside the sums of dQ.  The rows come in by way
// of LDS: loaded as operands, 32 bytes of each of 32 rows at a time, a training step of 16 x 616 tokens takes 380 us for 372.
template <int DP>
__global__ __launch_bounds__(ATT_THREADS, DP <= 64 ? 3 : 2) void attn_dq_kernel(const AttnArgs P, const AttnGrads G) {
    constexpr int TILE = DQ_KEYS * tile_row_bytes<DP>();
    __shared__ __align__(256) char smem[4 * TILE];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5;
    const int kvh = (int)blockIdx.x % P.Hkv, g = P.Hq / P.Hkv;
    SeqItem it;
    if (!locate_queries(P, lane, (int)blockIdx.x / P.Hkv, g, it)) return;
    const int item = it.item, q0 = it.q0, q1 = it.q1, k0 = it.k0, k1 = it.k1;
    const int nq = q1 - q0, nk = k1 - k0, ahead = nk - nq;
    const int units = (nq + ATT_ROWS - 1) / ATT_ROWS * g;
    const int first = units - 1 - item * ATT_WAVES, unit = first - wave;
    const int row0 = unit >= 0 ? unit / g * ATT_ROWS : 0, head = kvh * g + (unit >= 0 ? unit % g : 0);
    auto keys_of = [&](int row) { const int n = P.causal ? row + 1 + ahead : nk; return n < nk ? n : nk; };
    const int last = first / g * ATT_ROWS + ATT_ROWS;
    const int tiles = (max(keys_of((last < nq ? last : nq) - 1), 0) + DQ_KEYS - 1) / DQ_KEYS;
    const int wave_end = unit >= 0 ? keys_of((row0 + ATT_ROWS < nq ? row0 + ATT_ROWS : nq) - 1) : 0;
    const int all_see = keys_of(row0);
    const int row = row0 + (lane & 31);
    const bool row_ok = unit >= 0 && row < nq;
    const int row_keys = keys_of(row);

    const HeadRows K{P.k + kvh * P.k_head + (int64_t)k0 * P.k_tok, P.k_tok}, V{P.v + kvh * P.v_head + (int64_t)k0 * P.v_tok, P.v_tok};
    const uint32_t k_off = TileLoad<DP, DQ_KEYS>::first(tid, P.k_tok, P.D), v_off = TileLoad<DP, DQ_KEYS>::first(tid, P.v_tok, P.D);
    TileLoad<DP, DQ_KEYS> lk, lv;
    if (tiles > 0) {
        lk.load(K, 0, nk, P.D, k_off);
        lv.load(V, 0, nk, P.D, v_off);
    }
    bf16x8 qf[DP / 16], gf[DP / 16];
    float delta = 0.0f, lse = INFINITY;
    {
        const int64_t t = q0 + row0;
        const int rows = unit >= 0 ? min(nq - row0, ATT_ROWS) : 0;
        char* lds = smem + 2 * TILE + wave * 32 * tile_row_bytes<DP>();      // of the stage that is filled later
        RowsIn<DP> iq, ig, io;
        iq.load(P.q + head * P.q_head + t * P.q_tok, P.q_tok, rows, P.D, lane);
        ig.load(G.go + head * G.go_head + t * G.go_tok, G.go_tok, rows, P.D, lane);
        io.load(P.out + head * P.o_head + t * P.o_tok, P.o_tok, rows, P.D, lane);
        if (row_ok) lse = P.lse[(int64_t)head * P.Tq + q0 + row];
        bf16x8 of[DP / 16];
        iq.operands(lds, lane, qf);
        ig.operands(lds, lane, gf);
        io.operands(lds, lane, of);
#pragma unroll
        for (int d = 0; d < DP / 16; ++d) {
            float a[8], b[8];
            unpack_bf16x8(gf[d], a);
            unpack_bf16x8(of[d], b);
#pragma unroll
            for (int j = 0; j < 8; ++j) delta = fmaf(a[j], b[j], delta);
        }
        delta = halves_sum(delta);
    }
    const uint32_t rows_at = lds_addr_of(smem) + rows_lane<DP>(lane), cols_at = lds_addr_of(smem) + cols_lane<DP>(lane);
    f32x16 acc[DP / 32] = {};
    const float c = P.scale_log2;
    if (tiles > 0) {
        lk.store(smem, tid);
        lv.store(smem + TILE, tid);
    }
    __syncthreads();
    constexpr int N = DP / 16, NV = DP / 32;             // products of a score tile; of 16 keys with the columns
    if (wave_end > 0 && wave_end <= DQ_KEYS) {
        // Rows of few keys: out's rounding, which the sum over its columns carries into delta, would show in every dS of the row.  Their
        // keys are all in the first tile: delta = sum_j P_ij dP_ij.
        delta = 0.0f;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            f32x16 s = {}, dp = {};
#pragma unroll
            for (int d = 0; d < N; ++d) {
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_rows<DP>(rows_at, kb * 32, d), qf[d], s, 0, 0, 0);
                dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_rows<DP>(rows_at + TILE, kb * 32, d), gf[d], dp, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float w = __builtin_amdgcn_exp2f(fmaf(s[i], c, -lse)) * dp[i];
                delta += kb * 32 + 8 * (i >> 2) + 4 * h + (i & 3) < row_keys ? w : 0.0f;
            }
        }
        delta = halves_sum(delta);
    }
    if (row_ok && h == 0) G.delta[(int64_t)head * P.Tq + q0 + row] = delta;
    for (int t = 0; t < tiles; ++t) {
        const uint32_t stage = (uint32_t)(t & 1) * (2 * TILE), tk = rows_at + stage, tv = tk + TILE, tkc = cols_at + stage;
        if (t + 1 < tiles) {
            lk.load(K, (t + 1) * DQ_KEYS, nk, P.D, k_off);
            lv.load(V, (t + 1) * DQ_KEYS, nk, P.D, v_off);
        }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const int key0 = t * DQ_KEYS + kb * 32;
            if (key0 >= wave_end) continue;
            f32x16 s = {}, dp = {};
            constexpr int AHEAD = 3;
            bf16x8 f[AHEAD];
            auto operand = [&](int i) { return frag_rows<DP>(i < N ? tk : tv, kb * 32, i % N); };
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) f[i] = operand(i);
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int i = 0; i < 2 * N; ++i) {
                __builtin_amdgcn_sched_barrier(0);
                if (i < N) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % AHEAD], qf[i], s, 0, 0, 0);
                else dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % AHEAD], gf[i - N], dp, 0, 0, 0);
                if (i + AHEAD < 2 * N) f[i % AHEAD] = operand(i + AHEAD);
                if (i >= N) {
#pragma unroll
                    for (int e = (i - N) * 16 / N; e < (i - N + 1) * 16 / N; ++e) s[e] = __builtin_amdgcn_exp2f(fmaf(s[e], c, -lse));
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(0);
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] *= dp[i] - delta;
            if (key0 + 32 > all_see) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (key0 + 8 * (i >> 2) + 4 * h + (i & 3) >= row_keys) s[i] = 0.0f;
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const bf16x8 ds = pack_frag(s, k);
#pragma unroll
                for (int db = 0; db < NV; ++db)
                    acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_cols<DP>(tkc, kb * 32 + k * 16, db), ds, acc[db], 0, 0, 0);
            }
        }
        if (t + 1 < tiles) {
            char* nx = smem + ((t + 1) & 1) * 2 * TILE;
            lk.store(nx, tid);
            lv.store(nx + TILE, tid);
        }
        __syncthreads();
    }
    if (unit >= 0)
        store_rows<DP>(G.dq + head * G.dq_head + (int64_t)(q0 + row0) * G.dq_tok, G.dq_tok, min(nq - row0, ATT_ROWS), acc, P.scale, P.D, lane,
                       smem + wave * 32 * tile_row_bytes<DP>());
}

// ---- dK, dV: a wavefront has 32 keys and goes over the queries that see them, head by head of its group -------------------------
// The products leave a lane one key and 16 of 32 queries, so that the weights are the second operand of dV^T = dO^T P and dS of
// dK^T = Q^T dS.  The keys stay in registers beside the sums of dK and dV (160), the values in LDS: with both in registers the reloads of what
// is spilled wait for the tiles under way (1003 / 743 us at 4 x 2944 tokens).
constexpr int DKV_KEYS = ATT_WAVES * 32, DKV_ROWS = 32;

template <int DP>
__global__ __launch_bounds__(ATT_THREADS, DP <= 64 ? 3 : 2) void attn_dkv_kernel(const AttnArgs P, const AttnGrads G) {
    constexpr int ROWB = tile_row_bytes<DP>(), TILE = DKV_ROWS * ROWB, STAGE = 2 * TILE + 2 * DKV_ROWS * 4;
    __shared__ __align__(256) char smem[DKV_KEYS * ROWB + 2 * STAGE];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5;
    const int kvh = (int)blockIdx.x % P.Hkv, g = P.Hq / P.Hkv;
    SeqItem it;
    if (!locate_longest(P, lane, (int)blockIdx.x / P.Hkv, P.causal ? ATT_WAVES : 0, 1,
                        [](int nq, int nk, int& n, int& top) { n = (nk + DKV_KEYS - 1) / DKV_KEYS; top = (nq + 31) / 32; }, it))
        return;
    const int item = it.item, q0 = it.q0, q1 = it.q1, k0 = it.k0, k1 = it.k1;
    const int nq = q1 - q0, nk = k1 - k0, ahead = nk - nq;
    const int key0 = item * DKV_KEYS + wave * 32, key = key0 + (lane & 31);
    // row i sees key j if j <= i + ahead
    const int row_first = P.causal ? max(item * DKV_KEYS - ahead, 0) / DKV_ROWS : 0;
    const int row_tiles = max((nq + DKV_ROWS - 1) / DKV_ROWS - row_first, 0), steps = row_tiles * g;

    char* tv = smem;
    char* stage = smem + DKV_KEYS * ROWB;
    bf16x8 kf[DP / 16];
    {
        const HeadRows V{P.v + kvh * P.v_head + (int64_t)k0 * P.v_tok, P.v_tok};
        TileLoad<DP, DKV_KEYS> lv;
        lv.load(V, item * DKV_KEYS, nk, P.D, TileLoad<DP, DKV_KEYS>::first(tid, P.v_tok, P.D));
        load_rows<DP>(make_rsrc(P.k + kvh * P.k_head + (int64_t)(k0 + key0) * P.k_tok, 0x7fffffffu), (uint32_t)((lane & 31) * P.k_tok) * 2u,
                      key < nk, P.D, lane, kf);
        lv.store(tv, tid);
    }
    const uint32_t q_off = TileLoad<DP, DKV_ROWS>::first(tid, P.q_tok, P.D), g_off = TileLoad<DP, DKV_ROWS>::first(tid, G.go_tok, P.D);
    TileLoad<DP, DKV_ROWS> lq, lg;
    const float* row_stat = (wave & 1) != 0 ? G.delta : P.lse;       // the first wavefront loads the log-sum-exps, the second delta
    float stat = 0.0f;
    int tile_rows = 0;                                   // of the tile under way: the sequence's rows
    // step by step through the tiles of rows, the last first, head by head: of the next load, and of the tile in work
    const int r_last = (row_first + row_tiles - 1) * DKV_ROWS, r_first = row_first * DKV_ROWS;
    int head = kvh * g, load_r0 = r_last, r0 = r_last;
    auto load = [&]() {
        const int r0 = load_r0;
        lq.load(HeadRows{P.q + head * P.q_head + (int64_t)q0 * P.q_tok, P.q_tok}, r0, nq, P.D, q_off);
        lg.load(HeadRows{G.go + head * G.go_head + (int64_t)q0 * G.go_tok, G.go_tok}, r0, nq, P.D, g_off);
        tile_rows = min(nq - r0, DKV_ROWS);
        const __amdgpu_buffer_rsrc_t rs = make_rsrc(row_stat + (int64_t)head * P.Tq + q0 + r0, (uint32_t)tile_rows * 4u);
        stat = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rs, lane * 4, 0, 0));
        load_r0 -= DKV_ROWS;
        if (load_r0 < r_first) { load_r0 = r_last; ++head; }
    };
    auto store = [&](int n) {
        char* st = stage + (n & 1) * STAGE;
        lq.store(st, tid);
        lg.store(st + TILE, tid);
        // Rows past the sequence's: their log-sum-exp is infinity, so that their weights are 0 whatever q and grad_out read for them (0, or the last
        // row again where rows repeat or lie over one another); their delta is the 0 that it reads.  Here, not where it is loaded: there it would
        // wait for the tiles
        if (wave < 2 && lane < DKV_ROWS)
            reinterpret_cast<float*>(st + 2 * TILE)[wave * DKV_ROWS + lane] = wave == 0 && lane >= tile_rows ? INFINITY : stat;
    };
    const uint32_t v_at = lds_addr_of(tv) + (uint32_t)(wave * 32 * ROWB) + rows_lane<DP>(lane);
    const uint32_t rows_at = lds_addr_of(stage) + rows_lane<DP>(lane), cols_at = lds_addr_of(stage) + cols_lane<DP>(lane);
    f32x16 dk[DP / 32] = {}, dv[DP / 32] = {};
    const float c = P.scale_log2;
    if (steps > 0) {
        load();
        store(0);
    }
    __syncthreads();
    for (int n = 0; n < steps; ++n) {
        const uint32_t at = (uint32_t)(n & 1) * STAGE, tq = rows_at + at, tg = tq + TILE, tqc = cols_at + at, tgc = tqc + TILE;
        const float* st = reinterpret_cast<const float*>(stage + at + 2 * TILE);
        if (n + 1 < steps) load();
        auto work_on = [&]() {
            // Four times N products: scores, dP, dV, dK.  Operands are asked for AHEAD products before, the order is held, and the weights
            // lie beside dP's products, dS beside dV's.
            constexpr int N = DP / 16, NV = DP / 32, AHEAD = 2, VAHEAD = 2;
            auto operand = [&](int i) {
                const int j = i % N;
                switch (i / N) {
                    case 0: return frag_rows<DP>(tq, 0, j);
                    case 1: return frag_rows<DP>(tg, 0, j);
                    case 2: return frag_cols<DP>(tgc, j / NV * 16, j % NV);
                    default: return frag_cols<DP>(tqc, j / NV * 16, j % NV);
                }
            };
            auto four = [&](int at4) { return *reinterpret_cast<const f32x4*>(st + at4 + 4 * h); };      // of rows 8 q + 4 h ..: at4 = 8 q
            const int from = P.causal ? key - r0 - ahead - 4 * h : -1;   // the key is seen by the rows from it on
            f32x16 s = {}, dp = {};
            bf16x8 f[AHEAD], vf[VAHEAD], p[2], ds = {};
            f32x4 row4 = {};
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) f[i] = operand(i);
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int i = 0; i < 4 * N; ++i) {
                const int j = i % N, phase = i / N;
                __builtin_amdgcn_sched_barrier(0);
                if (i == 2 * N) {
                    p[0] = pack_frag(s, 0);
                    p[1] = pack_frag(s, 1);
                }
                if (phase == 3 && j % NV == 0) ds = pack_frag(s, j / NV);
                if (phase == 0) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % AHEAD], kf[j], s, 0, 0, 0);
                else if (phase == 1) dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % AHEAD], vf[j % VAHEAD], dp, 0, 0, 0);
                else if (phase == 2) dv[j % NV] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % AHEAD], p[j / NV], dv[j % NV], 0, 0, 0);
                else dk[j % NV] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % AHEAD], ds, dk[j % NV], 0, 0, 0);
                if (i + AHEAD < 4 * N) f[i % AHEAD] = operand(i + AHEAD);
                if (i >= N - VAHEAD && i < 2 * N - VAHEAD) vf[(i + VAHEAD) % VAHEAD] = frag_rows<DP>(v_at, 0, i + VAHEAD - N);
#pragma unroll
                for (int e = j * 16 / N; e < (j + 1) * 16 / N; ++e) {
                    if (phase == 1) {
                        if (e % 4 == 0) row4 = four(8 * (e / 4));
                        s[e] = __builtin_amdgcn_exp2f(fmaf(s[e], c, -row4[e % 4]));
                        if (8 * (e >> 2) + (e & 3) < from) s[e] = 0.0f;
                    }
                    if (phase == 2) {
                        if (e % 4 == 0) row4 = four(DKV_ROWS + 8 * (e / 4));
                        s[e] *= dp[e] - row4[e % 4];
                    }
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(0);
        };
        if (key0 < nk && (!P.causal || key0 <= min(r0 + DKV_ROWS, nq) - 1 + ahead)) {
            work_on();
        }
        if (n + 1 < steps) store(n + 1);
        __syncthreads();
        r0 = r0 == r_first ? r_last : r0 - DKV_ROWS;
    }
    if (key0 < nk) {
        char* rows = stage + wave * 32 * ROWB;           // every wavefront has read the last step's tiles
        const int n = min(nk - key0, 32);
        store_rows<DP>(G.dk + kvh * G.dk_head + (int64_t)(k0 + key0) * G.dk_tok, G.dk_tok, n, dk, P.scale, P.D, lane, rows);
        store_rows<DP>(G.dv + kvh * G.dv_head + (int64_t)(k0 + key0) * G.dv_tok, G.dv_tok, n, dv, 1.0f, P.D, lane, rows);
    }
}

static int64_t key_workgroups(const AttnArgs& a) { return ((int64_t)a.Tk / DKV_KEYS + a.n_seq) * a.Hkv; }

int64_t attn_backward_workgroups(int64_t Tq, int64_t Tk, int64_t n_seq, int64_t Hq, int64_t Hkv) {
    AttnArgs a{};
    a.Tq = (int)Tq; a.Tk = (int)Tk; a.n_seq = (int)n_seq; a.Hq = (int)Hq; a.Hkv = (int)Hkv;
    return std::max(attn_query_workgroups(a), key_workgroups(a));
}

hipError_t launch_attn_backward(const AttnArgs& a, const AttnGrads& gr, hipStream_t s) {
    const dim3 gq((uint32_t)attn_query_workgroups(a)), gk((uint32_t)key_workgroups(a));
    if (a.D <= 64) attn_dq_kernel<64><<<gq, ATT_THREADS, 0, s>>>(a, gr);
    else if (a.D <= 96) attn_dq_kernel<96><<<gq, ATT_THREADS, 0, s>>>(a, gr);
    else attn_dq_kernel<128><<<gq, ATT_THREADS, 0, s>>>(a, gr);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (a.D <= 64) attn_dkv_kernel<64><<<gk, ATT_THREADS, 0, s>>>(a, gr);
    else if (a.D <= 96) attn_dkv_kernel<96><<<gk, ATT_THREADS, 0, s>>>(a, gr);
    else attn_dkv_kernel<128><<<gk, ATT_THREADS, 0, s>>>(a, gr);
    return hipGetLastError();
}

}  // namespace skipffn
