// What the keys of packed prompts receive: w[kv head][j] = sum over the query heads of the group and the counted queries i that see j of
// P_ij = 2^(c q_i . k_j - lse_i), with the log-sum-exp that the forward saved, so that one product and one exponential a score is all.
//
// A wavefront owns 32 KW keys, which stay in registers as the product's first operand, and goes over the queries that see them, head by head of the
// group; tiles of 64 queries come through LDS, shared by the workgroup's wavefronts, two deep.  S^T = K Q^T leaves a lane one query and 16 of 32
// keys: its log-sum-exp is one number, and the sums of its keys stay in 16 registers until the end, where the lanes are joined.  No weight is
// rounded below fp32 and every sum has one owner and a fixed order.  Where keys are few for the chip, or a causal prompt's pieces uneven, the
// queries are cut into parts whose sums a second kernel adds.
//
// 32 / 8 heads of 128, us: 1 x 16384 tokens 1064-1127 by the card (975-1032 TFLOP/s of what the mask leaves, a library product of 8192^3 1178): matrix cores busy 48 % of the
// time, the vector unit 60 % (three instructions a score), at 2.0-2.1 GHz.  16 x up to 616 tokens 33, of which 4.3 the second kernel: latency, 1.2 a step of 64
// queries.  32768 keys by 64 queries 29-32 (67 MB of keys): loads and steps of a workgroup one after the other.
#include <algorithm>
#include <cmath>

#include "attn.hpp"

namespace skipffn {

// queries of a tile; sets of 32 keys of a wavefront (one: every operand of the queries is read for one product instead of two, and LDS is the bound: 1 x 16384
// tokens 1080 -> 1319 us, 16 x up to 616 the same); keys of a workgroup
constexpr int KW_ROWS = 64, KW = 2, KW_KEYS = ATT_WAVES * 32 * KW;

// keys of a workgroup, the longest pieces first
__device__ __forceinline__ bool locate_keys(const AttnArgs& P, const KeyWeightsArgs& W, int lane, int q, SeqItem& it) {
    return locate_longest(P, lane, q, P.causal && W.last >= P.Tq ? ATT_WAVES * KW : 0, 1,
                          [](int nq, int nk, int& n, int& top) { n = (nk + KW_KEYS - 1) / KW_KEYS; top = (nq + 31) / 32; }, it);
}

__device__ __forceinline__ void put_weight(const KeyWeightsArgs& W, int kvh, int key, float v) {
    float* w = W.w + kvh * W.w_head + key;
    *w = W.accumulate ? *w + v : v;
}

template <int DP>
__global__ __launch_bounds__(ATT_THREADS, 2) void attn_key_weights_kernel(const AttnArgs P, const KeyWeightsArgs W) {
    constexpr int ROWB = tile_row_bytes<DP>(), TILE = KW_ROWS * ROWB, STAGE = TILE + KW_ROWS * 4, N = DP / 16;
    __shared__ __align__(256) char smem[2 * STAGE];
    static_assert(2 * STAGE >= ATT_WAVES * 32 * ROWB, "a wavefront's keys come in by way of the stages");
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5;
    const int g = P.Hq / P.Hkv;
    int b = (int)blockIdx.x;
    const int kvh = b % P.Hkv; b /= P.Hkv;
    const int part = b % W.parts; b /= W.parts;
    SeqItem it;
    if (!locate_keys(P, W, lane, b, it)) return;
    const int nq = it.q1 - it.q0, nk = it.k1 - it.k0, ahead = nk - nq;
    const int key0 = it.item * KW_KEYS + wave * 32 * KW;           // of the wavefront
    // counted rows are base .. nq; row i sees key j if j <= i + ahead
    const int base = max(nq - W.last, 0), count = nq - base;
    const int tile0 = P.causal ? max(it.item * KW_KEYS - ahead - base, 0) / KW_ROWS : 0;
    const int steps = max((count + KW_ROWS - 1) / KW_ROWS - tile0, 0) * g;
    const int first = (int)((int64_t)steps * part / W.parts), last = (int)((int64_t)steps * (part + 1) / W.parts);

    const uint32_t q_off = TileLoad<DP, KW_ROWS>::first(tid, P.q_tok, P.D);
    TileLoad<DP, KW_ROWS> lq;
    float lse = 0.0f;
    int load_tile = tile0 + first / g, load_head = first % g;            // of the next load
    auto load = [&]() {
        const int head = kvh * g + load_head, row = base + load_tile * KW_ROWS;
        lq.load(HeadRows{P.q + head * P.q_head + (int64_t)it.q0 * P.q_tok, P.q_tok}, row, nq, P.D, q_off);
        if (tid < KW_ROWS) lse = row + tid < nq ? P.lse[(int64_t)head * P.Tq + it.q0 + row + tid] : 0.0f;
        if (++load_head == g) { load_head = 0; ++load_tile; }
    };
    auto store = [&](int n) {
        char* st = smem + (n & 1) * STAGE;
        lq.store(st, tid);
        if (tid < KW_ROWS) reinterpret_cast<float*>(st + TILE)[tid] = -lse;
    };
    if (first < last) load();                            // with the keys
    bf16x8 kf[KW][N];
    {
        char* lds = smem + wave * 32 * ROWB;
        const bf16_t* k = P.k + kvh * P.k_head + (int64_t)(it.k0 + key0) * P.k_tok;
        RowsIn<DP> in[KW];
#pragma unroll
        for (int i = 0; i < KW; ++i) in[i].load(k + (int64_t)i * 32 * P.k_tok, P.k_tok, min(nk - key0 - i * 32, 32), P.D, lane);
#pragma unroll
        for (int i = 0; i < KW; ++i) in[i].operands(lds, lane, kf[i]);
    }
    __syncthreads();

    float sum[KW][16] = {};
    const float c = P.scale_log2;
    const uint32_t rows_at = lds_addr_of(smem) + rows_lane<DP>(lane);
    int tile = tile0 + first / g, head = first % g;
    if (first < last) store(first);
    __syncthreads();
    for (int n = first; n < last; ++n) {
        if (n + 1 < last) load();
        const uint32_t at = rows_at + (uint32_t)(n & 1) * STAGE;
        const float* st = reinterpret_cast<const float*>(smem + (n & 1) * STAGE + TILE);
#pragma unroll
        for (int rb = 0; rb < KW_ROWS / 32; ++rb) {
            const int row0 = base + tile * KW_ROWS + rb * 32;
            const int seen = P.causal ? min(min(row0 + 32, nq) + ahead, nk) : nk;      // keys that the last row sees
            if (row0 >= nq || key0 >= seen) continue;
            float nl = st[rb * 32 + (lane & 31)];
            // operands a few products ahead of them
            constexpr int AHEAD = 3;
            bf16x8 f[AHEAD];
#pragma unroll
            for (int d = 0; d < AHEAD; ++d) f[d] = frag_rows<DP>(at, rb * 32, d);
            f32x16 s[KW];
#pragma unroll
            for (int i = 0; i < KW; ++i) s[i] = f32x16{};
#pragma unroll
            for (int d = 0; d < N; ++d) {
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < KW; ++i) s[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[i][d], f[d % AHEAD], s[i], 0, 0, 0);
                if (d + AHEAD < N) f[d % AHEAD] = frag_rows<DP>(at, rb * 32, d + AHEAD);
            }
            __builtin_amdgcn_sched_barrier(0);
            if (row0 + 32 > nq || (P.causal && key0 + 32 * KW > row0 + 1 + ahead)) {
                // Some rows are past the sequence's, or do not see some keys: minus infinity.  That is a weight of 0 beside a log-sum-exp that is a number; a
                // row with another one has NaN where it sees
                const int row = row0 + (lane & 31), keys = row >= nq ? 0 : P.causal ? row + 1 + ahead : nk;
                const bool number = fabsf(nl) < INFINITY;
#pragma unroll
                for (int i = 0; i < KW; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const bool sees = key0 + i * 32 + 8 * (e >> 2) + 4 * h + (e & 3) < keys;
                        s[i][e] = !sees ? -INFINITY : number ? s[i][e] : NAN;
                    }
                nl = number ? nl : 0.0f;
            }
#pragma unroll
            for (int i = 0; i < KW; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) sum[i][e] += __builtin_amdgcn_exp2f(fmaf(s[i][e], c, nl));
        }
        if (n + 1 < last) store(n + 1);
        __syncthreads();
        if (++head == g) { head = 0; ++tile; }
    }
    // Over the 32 lanes of a half: each exchange halves the registers, lane bit 4 - k tells which half stays
#pragma unroll
    for (int i = 0; i < KW; ++i) {
        float* v = sum[i];
#pragma unroll
        for (int off = 16, m = 8; m > 0; off >>= 1, m >>= 1) {
            const bool up = (lane & off) != 0;
#pragma unroll
            for (int e = 0; e < m; ++e) {
                const float send = up ? v[e] : v[e + m], keep = up ? v[e + m] : v[e];
                v[e] = keep + __shfl_xor(send, off, 64);
            }
        }
        const float w = v[0] + __shfl_xor(v[0], 1, 64);
        const int e = (lane >> 1) & 15, key = key0 + i * 32 + 8 * (e >> 2) + 4 * h + (e & 3);
        if ((lane & 1) == 0 && key < nk) {
            if (W.parts > 1) W.part[((int64_t)part * P.Hkv + kvh) * P.Tk + it.k0 + key] = w;
            else put_weight(W, kvh, it.k0 + key, w);
        }
    }
}

// the parts' sums, added in order
__global__ __launch_bounds__(KW_KEYS) void key_weights_join_kernel(const AttnArgs P, const KeyWeightsArgs W) {
    const int kvh = (int)blockIdx.x % P.Hkv;
    SeqItem it;
    if (!locate_keys(P, W, threadIdx.x & 63, (int)blockIdx.x / P.Hkv, it)) return;
    const int key = it.k0 + it.item * KW_KEYS + (int)threadIdx.x;
    if (key >= it.k1) return;
    const float* p = W.part + (int64_t)kvh * P.Tk + key;
    float v = 0.0f;
    for (int z = 0; z < W.parts; ++z) v += p[(int64_t)z * P.Hkv * P.Tk];
    put_weight(W, kvh, key, v);
}

// Parts that the queries are cut into.  A piece takes 1.2 us a step and 6 us to begin and end; the last ones leave the chip to themselves, so pieces are made
// shorter until what that saves goes into beginning more of them; the second kernel takes about 4 us.  Us of whole
// calls (parts), as planned first: 16 sequences of up to 616, 5682 tokens together, 34.6 (3), 60.8 (1), 40.1 (6); 8 x 616 37.0 (4), 67.3 (1), 45.3 (2), 45.0 (9); 1 x 616 16.6 (10, all there
// are), 65.4 (1), 19.4 (7); 1 x 2944 56.7 (14), 257 (1), 59.5 (7), 69.7 (28); 4 x 4096 324 (7), 397 (1), 316 (3), 363 (14); 1 x 16384 1074 (14), 1501 (1), 1059 (7), 1134 (28)
KeyWeightsPlan key_weights_plan(int64_t Tq, int64_t Tk, int64_t n_seq, int64_t Hq, int64_t Hkv, int64_t last, int ncu) {
    KeyWeightsPlan p{};
    p.blocks = (Tk / KW_KEYS + n_seq) * Hkv;
    const int64_t rows = n_seq > 0 ? std::min(Tq / n_seq, last) : 0, steps = (rows + KW_ROWS - 1) / KW_ROWS * (Hq / Hkv);
    const double piece = 1.2 * (double)steps, begin = 6.0 * (double)p.blocks / (2.0 * ncu);
    // a launch has fewer than 2^24 workgroups
    const int64_t fit = (((int64_t)1 << 24) - 1) / std::max<int64_t>(p.blocks, 1);
    const int64_t parts = std::min<int64_t>({steps / 4, (int64_t)std::lround(std::sqrt(piece / std::max(begin, 1e-3))), KEY_WEIGHTS_MAX_PARTS, fit});
    p.parts = parts > 1 && piece - piece / (double)parts > 5.0 ? (int)parts : 1;
    return p;
}

template <int DP>
static void launch_kw(const AttnArgs& a, const KeyWeightsArgs& w, const KeyWeightsPlan& p, hipStream_t s) {
    attn_key_weights_kernel<DP><<<(uint32_t)(p.blocks * p.parts), ATT_THREADS, 0, s>>>(a, w);
}

hipError_t launch_attn_key_weights(const AttnArgs& a, const KeyWeightsArgs& w, const KeyWeightsPlan& p, hipStream_t s) {
    if (a.D <= 64) launch_kw<64>(a, w, p, s);
    else if (a.D <= 96) launch_kw<96>(a, w, p, s);
    else launch_kw<128>(a, w, p, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.parts == 1) return e;
    key_weights_join_kernel<<<(uint32_t)p.blocks, KW_KEYS, 0, s>>>(a, w);
    return hipGetLastError();
}

}  // namespace skipffn
