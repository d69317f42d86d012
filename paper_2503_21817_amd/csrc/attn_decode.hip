// Attention of single new tokens over a cache: the rows of the prefix that the sequences of a group share, then each sequence's own.
//
// The rows of a product are (sequence, query head) pairs: as many sequences of a group as fill 32 rows with the heads of one
// key/value head, so that a prefix is read once for all of them.  Their keys are one list of tiles of 32: the prefix's, seen by
// every row, then each sequence's own, seen by its rows alone.  The list is cut into `splits` even parts, one a workgroup, and
// a part is dealt out to the four wavefronts, each with tiles of its own in LDS (nothing is waited for but a wavefront's own loads);
// the wavefronts' maxima, sums and rows are joined in LDS, those of the parts by a second kernel.  Few rows of a product are in use
// where little is shared (4 of 32 with 32 / 8 heads and no sharing): the matrix cores have the time, the reads of the cache bound it.
//
// Measured, 32 / 8 heads of 128, us: 4 caches of up to 32768 rows (300 MB) 62-65 where the inputs change from pass to pass, 4.6-4.8 TB/s (a large
// copy: 5.0), of which the second kernel 4.3; 64 sequences on two prefixes of up to 5795 rows (54 MB) 18.4-19.1 + 4: some tiles a wavefront one after
// the other, a latency each; 8 sequences of 184 + 64 rows 8.1-8.8, all latency.
#include <algorithm>

#include "attn.hpp"

namespace skipffn {

constexpr int DEC_KEYS = 32;

template <int DP>
__global__ __launch_bounds__(ATT_THREADS, DP <= 64 ? 3 : 2) void attn_decode_kernel(const AttnDecodeArgs P) {
    constexpr int ROWB = tile_row_bytes<DP>(), TILE = DEC_KEYS * ROWB;
    static_assert(2 * TILE >= DP * 32 * 4, "a wavefront's sums fit where its tiles were");
    __shared__ __align__(256) char smem[ATT_WAVES * 2 * TILE];
    __shared__ float stat[ATT_WAVES][2][32];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5;
    const int g = P.Hq / P.Hkv, members = g >= 32 ? 1 : 32 / g, head_blocks = (g + 31) / 32;
    // blockIdx.x: key/value head, then block of its query heads, then sequences; blockIdx.y: part
    int b = (int)blockIdx.x;
    const int kvh = b % P.Hkv; b /= P.Hkv;
    const int hb = b % head_blocks; b /= head_blocks;
    // Which sequences: a lane takes a group (the one past the last: the sequences of none), a prefix sum over the lanes finds the workgroup's.
    // What depends on the group is loaded with its bounds, and so are the lengths if a wavefront holds them all: one latency, not three.
    const bool few = P.n_seq <= 64;
    const int all_own = few && lane < P.n_seq && P.cap > 0 ? P.suffix_len[lane] : 0;
    int s0 = 0, ns = 0, p0 = 0, p1 = 0;
    for (int i0 = 0, before = 0; i0 <= P.n_groups; i0 += 64) {
        const int i = i0 + lane;
        int lo = 0, hi = 0, pb = 0, pe = 0;
        if (i < P.n_groups) {
            seg_bounds(P.group_off, i, P.n_seq, lo, hi);
            if (P.Tp > 0) seg_bounds(P.prefix_seg, i, P.Tp, pb, pe);
        } else if (i == P.n_groups) {
            lo = P.n_groups > 0 ? min(max(P.group_off[P.n_groups], 0), P.n_seq) : 0;
            hi = P.n_seq;
        }
        const int n = (hi - lo + members - 1) / members, incl = wave_inclusive_sum(n);
        const uint64_t past = __ballot(b < before + incl);
        if (past != 0) {
            const int l = __builtin_ctzll(past);
            s0 = __builtin_amdgcn_readlane(lo, l) + (b - before - __builtin_amdgcn_readlane(incl - n, l)) * members;
            ns = min(__builtin_amdgcn_readlane(hi, l) - s0, members);
            p0 = __builtin_amdgcn_readlane(pb, l);
            p1 = __builtin_amdgcn_readlane(pe, l);
            break;
        }
        before += __builtin_amdgcn_readlane(incl, 63);
    }
    if (ns == 0) return;
    const int heads = min(g - hb * 32, 32), rows = ns * heads;
    const int prefix_tiles = (p1 - p0 + DEC_KEYS - 1) / DEC_KEYS;
    // lane i: own keys of sequence s0 + i and the tiles up to it
    int own_keys = 0;
    if (few) own_keys = __shfl(all_own, s0 + lane, 64);
    else if (lane < ns && P.cap > 0) own_keys = P.suffix_len[s0 + lane];
    own_keys = lane < ns ? min(max(own_keys, 0), P.cap) : 0;
    const int own_tiles = (own_keys + DEC_KEYS - 1) / DEC_KEYS, own_sum = wave_inclusive_sum(own_tiles);
    const int tiles = prefix_tiles + __builtin_amdgcn_readlane(own_sum, 63);
    const int z = (int)blockIdx.y;
    const int t_first = (int)((int64_t)tiles * z / P.splits) + wave, t_end = (int)((int64_t)tiles * (z + 1) / P.splits);

    const int r = lane & 31, member = r / heads, head = kvh * g + hb * 32 + r % heads;
    bf16x8 qf[DP / 16];
    load_rows<DP>(make_rsrc(P.q + (int64_t)s0 * P.q_tok + (int64_t)(kvh * g + hb * 32) * P.q_head, 0x7fffffffu),
                  (uint32_t)(member * P.q_tok + (r % heads) * (int)P.q_head) * 2u, r < rows, P.D, lane, qf);

    char* tk = smem + wave * 2 * TILE;
    char* tv = tk + TILE;
    const uint32_t rows_at = lds_addr_of(tk) + rows_lane<DP>(lane), cols_at = lds_addr_of(tv) + cols_lane<DP>(lane);
    typedef TileLoad<DP, DEC_KEYS, 64> Load;
    const uint32_t pk_off = Load::first(lane, P.pk_tok, P.D), pv_off = Load::first(lane, P.pv_tok, P.D);
    const uint32_t sk_off = Load::first(lane, P.sk_tok, P.D), sv_off = Load::first(lane, P.sv_tok, P.D);
    Load lk, lv;
    int next_keys = 0, next_of = -1;                     // of the tile under way: its keys, and whose they are (-1: all rows')
    bool dropped = false, seen = false;                  // seen: the row sees a key of the wavefront's
    auto own_tile = [&](int u, int& i, int& k0, int& n) {    // member, first key, its keys
        i = __builtin_ctzll(__ballot(u < own_sum));
        k0 = (u - __builtin_amdgcn_readlane(own_sum - own_tiles, i)) * DEC_KEYS;
        n = __builtin_amdgcn_readlane(own_keys, i);
    };
    auto load = [&](int t) {
        if (t < prefix_tiles) {
            next_of = -1;
            next_keys = min(p1 - p0 - t * DEC_KEYS, DEC_KEYS);
            lk.load(HeadRows{P.pk + kvh * P.pk_head + (int64_t)p0 * P.pk_tok, P.pk_tok}, t * DEC_KEYS, p1 - p0, P.D, pk_off);
            lv.load(HeadRows{P.pv + kvh * P.pv_head + (int64_t)p0 * P.pv_tok, P.pv_tok}, t * DEC_KEYS, p1 - p0, P.D, pv_off);
        } else {
            int i, k0, n;
            own_tile(t - prefix_tiles, i, k0, n);
            next_of = i;
            next_keys = min(n - k0, DEC_KEYS);
            lk.load(HeadRows{P.sk + (s0 + i) * P.sk_seq + kvh * P.sk_head, P.sk_tok}, k0, n, P.D, sk_off);
            lv.load(HeadRows{P.sv + (s0 + i) * P.sv_seq + kvh * P.sv_head, P.sv_tok}, k0, n, P.D, sv_off);
        }
    };
    f32x16 acc[DP / 32] = {};
    float m = -INFINITY, l = 0.0f;
    const float c = P.scale_log2;
    if (t_first < t_end) load(t_first);
    for (int t = t_first; t < t_end; t += ATT_WAVES) {
        const int keys = next_keys;
        // a wavefront's LDS operations are done in order: its last tile has been read
        // Own rows of one sequence come to the others' with weight 0, which would make a NaN of an infinity or a NaN: these leave the tile,
        // and are added to the rows that see them at the end
        if (next_of >= 0 && ns > 1 && __ballot(lv.any_not_finite()) != 0) {
            lv.drop_not_finite();
            dropped = true;
        }
        const bool sees = next_of < 0 || member == next_of;
        seen |= sees;
        lk.store(tk, lane);
        lv.store(tv, lane);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (t + ATT_WAVES < t_end) load(t + ATT_WAVES);
        // operands a few products ahead of them and the order held, as in the kernels over whole prompts
        constexpr int N = DP / 16, NV = DP / 32, AHEAD = 3, VAHEAD = 2;
        f32x16 s = {};
        bf16x8 f[AHEAD], vf[VAHEAD], p = {};
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) f[i] = frag_rows<DP>(rows_at, 0, i);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            __builtin_amdgcn_sched_barrier(0);
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % AHEAD], qf[i], s, 0, 0, 0);
            if (i + AHEAD < N) f[i % AHEAD] = frag_rows<DP>(rows_at, 0, i + AHEAD);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (keys < DEC_KEYS) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (8 * (i >> 2) + 4 * h + (i & 3) >= keys) s[i] = -INFINITY;
        }
        float top = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
        top = sees ? halves_max(top) : -INFINITY;
        // the maximum may lag, as in the kernels over whole prompts, and each row by its own scores
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
        auto weights = [&](int i0) {
#pragma unroll
            for (int i = i0; i < i0 + 8; ++i) {
                s[i] = sees ? __builtin_amdgcn_exp2f(fmaf(s[i], c, -mc)) : 0.0f;
                l += s[i];
            }
        };
#pragma unroll
        for (int i = 0; i < VAHEAD; ++i) vf[i] = frag_cols<DP>(cols_at, i / NV * 16, i % NV);
        weights(0);
#pragma unroll
        for (int i = 0; i < 2 * NV; ++i) {
            __builtin_amdgcn_sched_barrier(0);
            if (i % NV == 0) p = pack_frag(s, i / NV);
            acc[i % NV] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[i % VAHEAD], p, acc[i % NV], 0, 0, 0);
            if (i + VAHEAD < 2 * NV) vf[i % VAHEAD] = frag_cols<DP>(cols_at, (i + VAHEAD) / NV * 16, (i + VAHEAD) % NV);
            if (i == 0) weights(8);
        }
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    if (dropped) {
        for (int t = t_first; t < t_end; t += ATT_WAVES) {
            const int u = t - prefix_tiles;
            if (u < 0) continue;
            int i, k0, n;
            own_tile(u, i, k0, n);
            const bf16_t* v = P.sv + (s0 + i) * P.sv_seq + kvh * P.sv_head + (int64_t)k0 * P.sv_tok;
            for (int j = min(n - k0, DEC_KEYS); j > 0; --j, v += P.sv_tok) add_not_finite<DP>(acc, v, P.D, h, member == i);
        }
    }
    // join the wavefronts: [column][row] of each where its tiles were
    l = halves_sum(l);
    if (seen) m = fmaxf(m, -FLT_MAX);                    // minus infinity: no key, as in attn_join.hip
    float* mine = reinterpret_cast<float*>(tk);
#pragma unroll
    for (int db = 0; db < DP / 32; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) mine[(db * 32 + 8 * (i >> 2) + 4 * h + (i & 3)) * 32 + r] = acc[db][i];
    if (h == 0) {
        stat[wave][0][r] = m;
        stat[wave][1][r] = l;
    }
    __syncthreads();
    constexpr int PER = DP / 8;                          // columns of a thread: eight threads a row
    const int jr = tid & 31, jd = (tid >> 5) * PER;
    if (jr >= rows) return;
    float top = -INFINITY, w[ATT_WAVES], sum = 0.0f, o[PER];
#pragma unroll
    for (int i = 0; i < ATT_WAVES; ++i) top = fmaxf(top, stat[i][0][jr]);
#pragma unroll
    for (int i = 0; i < ATT_WAVES; ++i) {
        w[i] = stat[i][0][jr] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((stat[i][0][jr] - top) * c);
        sum += w[i] * stat[i][1][jr];
    }
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        o[j] = 0.0f;
#pragma unroll
        for (int i = 0; i < ATT_WAVES; ++i) o[j] = fmaf(w[i], reinterpret_cast<const float*>(smem + i * 2 * TILE)[(jd + j) * 32 + jr], o[j]);
    }
    const int seq = s0 + jr / heads, hq = kvh * g + hb * 32 + jr % heads;
    if (P.splits > 1) {
        const int64_t at = ((int64_t)seq * P.Hq + hq) * P.splits + z;
        if (jd == 0) {
            P.stat[2 * at] = top;
            P.stat[2 * at + 1] = sum;
        }
#pragma unroll
        for (int j = 0; j < PER; j += 4) *reinterpret_cast<f32x4*>(P.part + at * attn_padded_columns(DP) + jd + j) = f32x4{o[j], o[j + 1], o[j + 2], o[j + 3]};
        return;
    }
    const float inv = top == -INFINITY ? 0.0f : 1.0f / sum;   // a row that sees no key is zero
    bf16_t* out = P.out + (int64_t)seq * P.o_tok + hq * P.o_head;
#pragma unroll
    for (int j = 0; j < PER; j += 4)
        if (jd + j < P.D)
            *reinterpret_cast<u32x2*>(out + jd + j) =
                u32x2{pack_bf16x2(o[j] * inv, o[j + 1] * inv), pack_bf16x2(o[j + 2] * inv, o[j + 3] * inv)};
}

namespace {
int64_t decode_blocks(int64_t n_seq, int64_t n_groups, int64_t Hq, int64_t Hkv) {
    const int64_t g = Hq / Hkv, members = g >= 32 ? 1 : 32 / g;
    // the sum of ceil(n / members) over the groups and the sequences of none
    return std::min(n_seq, n_seq / members + n_groups + 1) * Hkv * ((g + 31) / 32);
}
}  // namespace

// As many parts as give every compute unit two workgroups (one / two / three, us: 64 sequences on 2 prefixes of up to 5795 rows 25.5 / 23.3 / 29.3,
// 128 on 2 of 1000 29.2 / 24.5 / 32.5, 4 caches of up to 32768 rows 64 / 65 / 66), but none of fewer than 192 keys of the longest list that the
// bounds allow on average (128 / 256, us: 1 sequence of 600 + 100 rows 9.0 / 10.2, 8 of 184 + 64 9.9 / 8.3)
int attn_decode_splits(int64_t n_seq, int64_t n_groups, int64_t Hq, int64_t Hkv, int64_t Tp, int64_t cap, int ncu) {
    if (n_seq <= 0) return 1;
    const int64_t g = Hq / Hkv, members = g >= 32 ? 1 : 32 / g;
    const int64_t blocks = std::max<int64_t>(std::max(n_groups, (n_seq + members - 1) / members), 1) * Hkv * ((g + 31) / 32);
    const int64_t shared = std::max<int64_t>(1, std::min(members, n_groups > 0 ? n_seq / n_groups : members));
    const int64_t keys = (n_groups > 0 ? Tp / n_groups : 0) + shared * cap;
    const int64_t want = (2 * (int64_t)ncu + blocks - 1) / blocks, most = keys * 2 / (DEC_KEYS * ATT_WAVES * 3);
    return (int)std::max<int64_t>(1, std::min<int64_t>(std::min(want, most), ATTN_MAX_SPLITS));
}

hipError_t launch_attn_decode(const AttnDecodeArgs& a, hipStream_t s) {
    const dim3 grid((uint32_t)decode_blocks(a.n_seq, a.n_groups, a.Hq, a.Hkv), (uint32_t)a.splits);
    if (a.D <= 64) attn_decode_kernel<64><<<grid, ATT_THREADS, 0, s>>>(a);
    else if (a.D <= 96) attn_decode_kernel<96><<<grid, ATT_THREADS, 0, s>>>(a);
    else attn_decode_kernel<128><<<grid, ATT_THREADS, 0, s>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    AttnJoinArgs j{};
    j.T = a.n_seq; j.Hq = a.Hq; j.D = a.D; j.splits = a.splits; j.scale_log2 = a.scale_log2;
    j.part = a.part; j.stat = a.stat;
    j.out = a.out; j.o_tok = a.o_tok; j.o_head = a.o_head;
    return launch_attn_join(j, s);
}

}  // namespace skipffn
