// What queries and keys get between the projection and the attention: an RMS norm of each head (optional) and the rotation of pairs of
// columns by angles position x frequency, in one pass over them; the values of the same tokens go into the cache with it.
//     n = x rsqrt(mean x^2 + eps) gain,   (y_a, y_b) = (n_a cos - n_b sin, n_a sin + n_b cos)
// Backward: the gradient is rotated back, and with r = rsqrt(mean x^2 + eps), g the rotated gradient:
//     d_gain = sum g x r,   dx = r (g gain - x r^2 mean(g gain x))
// All in fp32, rounded once where a result leaves.
//
// A lane has two slots of V columns of a head, the two that are rotated together: columns c and c + rot / 2 of the halves, or neighbours.  LPH lanes
// share a head (their sums of squares are joined by exchanges), a wavefront works on several heads of a token, so that the V angles of a lane are
// taken once for all of them.  An angle is the product in 64 bits (a position of 10^6 leaves 32 bits an error of 0.06 radians), brought to
// [-1/2, 1/2] turns there; sine and cosine are v_sin_f32 and v_cos_f32, off by 2^-22.9 at most over that range (compared with 64 bits at 2^24 places).
#include <algorithm>
#include <type_traits>

#include "colsum.hpp"
#include "kernels.hpp"

namespace skipffn {

constexpr int ROPE_THREADS = 256, ROPE_WAVES = ROPE_THREADS / 64;

// V columns: 8 (16 bytes), or 4 where the halves of the rotated columns are not whole 16 bytes
template <int V> struct RopeVec;
template <> struct RopeVec<8> { typedef u32x4 type; };
template <> struct RopeVec<4> { typedef u32x2 type; };

template <int V>
__device__ __forceinline__ void rope_unpack(const typename RopeVec<V>::type& v, float* f) {
#pragma unroll
    for (int j = 0; j < V / 2; ++j) {
        f[2 * j] = bf16lo_to_f32(v[j]);
        f[2 * j + 1] = bf16hi_to_f32(v[j]);
    }
}
template <int V>
__device__ __forceinline__ typename RopeVec<V>::type rope_pack(const float* f) {
    typename RopeVec<V>::type v;
#pragma unroll
    for (int j = 0; j < V / 2; ++j) v[j] = pack_bf16x2(f[2 * j], f[2 * j + 1]);
    return v;
}

// Where a lane's two slots lie in a head, and whether they are rotated; a slot past the head has no columns
template <int V, int LPH, bool PAIRS>
struct RopeLane {
    int u, col[2];
    bool has[2], turned[2];
    __device__ __forceinline__ RopeLane(int lane, int D, int rot) {
        u = lane % LPH;
        const int half = rot / 2 / V;                    // slots of half of the rotated columns
        int a = 2 * u, b = 2 * u + 1;
        if (!PAIRS && u < half) {
            a = u;
            b = u + half;
        }
        col[0] = a * V;
        col[1] = b * V;
        has[0] = col[0] < D;
        has[1] = col[1] < D;
        turned[0] = PAIRS ? col[0] < rot : u < half;
        turned[1] = PAIRS ? col[1] < rot : u < half;
    }
    // the lane's frequencies u V + i, and their axes, two bits each
    float freq[V];
    uint32_t axes;
    __device__ __forceinline__ void frequencies(const RopeArgs& P) {
        axes = 0;
#pragma unroll
        for (int i = 0; i < V; ++i) freq[i] = 0.0f;
        if (P.rot == 0) return;
        // every load is made, of the last frequency where the lane has none: as branches they would wait for one another
#pragma unroll
        for (int i = 0; i < V; ++i) freq[i] = P.inv_freq[min(u * V + i, P.rot / 2 - 1)];
        if (P.n_axes > 1) {
#pragma unroll
            for (int w = 0; w < V / 4; ++w) {
                const uint32_t four = *reinterpret_cast<const uint32_t*>(P.axis + u * V + w * 4);
                axes |= ((four & 3) | (four >> 6 & 0xc) | (four >> 12 & 0x30) | (four >> 18 & 0xc0)) << (8 * w);
            }
        }
    }
    // positions of a token
    struct Place { int32_t pos[ROPE_MAX_AXES]; };
    static __device__ __forceinline__ Place place(const RopeArgs& P, int t) {
        Place p;
#pragma unroll
        for (int a = 0; a < ROPE_MAX_AXES; ++a) p.pos[a] = 0;
        if (P.n_axes > 0) p.pos[0] = P.pos[t];
        if (P.n_axes > 1) {
#pragma unroll
            for (int a = 1; a < ROPE_MAX_AXES; ++a) p.pos[a] = P.pos[(int64_t)min(a, P.n_axes - 1) * P.T + t];
        }
        return p;
    }
    // cosine and sine of the frequencies' angles there
    __device__ __forceinline__ void angles(const Place& at, float (&cs)[V], float (&sn)[V]) const {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int axis = axes >> (2 * i) & 3;
            int32_t p = at.pos[0];
#pragma unroll
            for (int a = 1; a < ROPE_MAX_AXES; ++a) p = axis == a ? at.pos[a] : p;
            const double x = (double)p * (double)freq[i] * 0.15915494309189533577;       // in turns
            const float f = (float)(x - rint(x));
            sn[i] = __builtin_amdgcn_sinf(f);
            cs[i] = __builtin_amdgcn_cosf(f);
        }
    }
    // (x_a, x_b) rotated by the angles, or by their opposites
    __device__ __forceinline__ void rotate(float* xa, float* xb, const float (&cs)[V], const float (&sn)[V], bool back) const {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if constexpr (PAIRS) {
                float* x = i < V / 2 ? xa + 2 * i : xb + 2 * (i - V / 2);
                const float s = back ? -sn[i] : sn[i], p = x[0] * cs[i] - x[1] * s, q = x[0] * s + x[1] * cs[i];
                const bool turn = turned[i < V / 2 ? 0 : 1];
                x[0] = turn ? p : x[0];
                x[1] = turn ? q : x[1];
            } else {
                const float s = back ? -sn[i] : sn[i], p = xa[i] * cs[i] - xb[i] * s, q = xa[i] * s + xb[i] * cs[i];
                xa[i] = turned[0] ? p : xa[i];
                xb[i] = turned[0] ? q : xb[i];
            }
        }
    }
};

// over the LPH lanes of a head: neighbours, pairs, then mirrored halves of 8 and 16 lanes, whose quarters and halves agree by then
template <int LPH>
__device__ __forceinline__ float head_sum(float v) {
    auto add = [&](auto ctrl) {
        v += __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), decltype(ctrl)::value, 0xF, 0xF, false));
    };
    add(std::integral_constant<int, 0xB1>{});            // quad_perm 1, 0, 3, 2
    add(std::integral_constant<int, 0x4E>{});            // quad_perm 2, 3, 0, 1
    if constexpr (LPH >= 8) add(std::integral_constant<int, 0x141>{});
    if constexpr (LPH >= 16) add(std::integral_constant<int, 0x140>{});
    return v;
}
// a slot of a head's columns; one past its columns reads the first and is 0
template <int V>
__device__ __forceinline__ typename RopeVec<V>::type rope_slot(const bf16_t* head, int col, bool has) {
    typedef typename RopeVec<V>::type Vec;
    const Vec v = *reinterpret_cast<const Vec*>(head + (has ? col : 0));
    return has ? v : Vec{};
}

// Heads that a wavefront has at a time, and tokens beside one another: powers of two whose product with LPH is 64
__host__ __device__ inline int rope_heads_at_once(int lph, int heads) {
    int n = 1;
    while (n * 2 * lph <= 64 && n < heads) n *= 2;
    return n;
}

// A wavefront has U times as many heads of its tokens as it works on at once; all of their loads are asked for first.
// Bound by bytes: 11776 tokens of 32 / 8 heads of 128 with their values into a cache 59.5-60.5 us (290 MB, 4.8 TB/s; a large copy 4.9), 9856 with the norm 49.8
// (202 MB).  With loads under branches, which wait for one another, 68; with sincospif instead of the two instructions 74.
template <int V, int LPH, int U, bool PAIRS, bool NORM>
__global__ __launch_bounds__(ROPE_THREADS) void rope_fwd_kernel(const RopeArgs P, const int chunks) {
    typedef typename RopeVec<V>::type Vec;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int heads = P.Hq + P.Hkv + (P.v.p != nullptr ? P.Hkv : 0), at_once = rope_heads_at_once(LPH, heads), tokens = 64 / LPH / at_once;
    const int64_t unit = (int64_t)blockIdx.x * ROPE_WAVES + wave;
    const int64_t group = unit / chunks;
    const int chunk = (int)(unit - group * chunks);
    const int64_t t64 = group * tokens + lane / (LPH * at_once);
    if (t64 >= P.T) return;
    const int t = (int)t64;
    RopeLane<V, LPH, PAIRS> L(lane, P.D, P.rot);
    L.frequencies(P);
    const auto place = L.place(P, t);
    const int64_t row = P.row != nullptr ? (int64_t)P.row[t] : t;
    const bool stored = row >= 0 && row < P.rows_out;    // of k and v
    int head[U];
    bf16_t* to[U];
    Vec x[U][2];
#pragma unroll
    for (int i = 0; i < U; ++i) {
        head[i] = (chunk * U + i) * at_once + lane / LPH % at_once;
        // what goes nowhere reads the token's first query
        const bool is_q = head[i] < P.Hq, goes = is_q || (head[i] < heads && stored), is_k = !is_q && head[i] < P.Hq + P.Hkv;
        const int h = is_q ? head[i] : is_k ? head[i] - P.Hq : head[i] - P.Hq - P.Hkv;
        const RopeIn from = is_q || !goes ? P.q : is_k ? P.k : P.v;
        const RopeOut out = is_q ? P.q_out : is_k ? P.k_out : P.v_out;
        to[i] = goes ? out.p + (is_q ? (int64_t)t : row) * out.tok + h * out.head : nullptr;
#pragma unroll
        for (int j = 0; j < 2; ++j) x[i][j] = rope_slot<V>(from.p + (int64_t)t * from.tok + (goes ? h : 0) * from.head, L.col[j], L.has[j]);
    }
    float cs[V], sn[V];
    L.angles(place, cs, sn);
#pragma unroll
    for (int i = 0; i < U; ++i) {
        if (head[i] < P.Hq + P.Hkv) {
            float a[V], b[V];
            rope_unpack<V>(x[i][0], a);
            rope_unpack<V>(x[i][1], b);
            if constexpr (NORM) {
                float ss = 0.0f;
#pragma unroll
                for (int j = 0; j < V; ++j) ss = fmaf(a[j], a[j], fmaf(b[j], b[j], ss));
                const float r = rsqrtf(head_sum<LPH>(ss) * P.inv_D + P.eps);
                const bf16_t* gain = head[i] < P.Hq ? P.gain_q : P.gain_k;
                float ga[V], gb[V];
                if (gain != nullptr) {
                    rope_unpack<V>(rope_slot<V>(gain, L.col[0], L.has[0]), ga);
                    rope_unpack<V>(rope_slot<V>(gain, L.col[1], L.has[1]), gb);
                }
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    a[j] *= gain != nullptr ? r * ga[j] : r;
                    b[j] *= gain != nullptr ? r * gb[j] : r;
                }
            }
            L.rotate(a, b, cs, sn, false);
            x[i][0] = rope_pack<V>(a);
            x[i][1] = rope_pack<V>(b);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j)
            if (to[i] != nullptr && L.has[j]) *reinterpret_cast<Vec*>(to[i] + L.col[j]) = x[i][j];
    }
}

// A workgroup has either heads of q or heads of k and goes on through the tokens; the next heads' loads are under way while these are worked on.  With gain
// gradients every lane keeps the sums of its columns, joined over the workgroup at the end: part [workgroup][D], q's first.
// Bound by bytes: 9856 tokens of 32 / 8 heads of 128 with both gains 58.9 us (303 MB, 5.1 TB/s), the gains' second kernel 4.8; forward and backward 111.  Without
// the loads asked for early, heads of q and k in one workgroup and gains read where they are used 225; two heads at a time 144 (197 registers); four
// workgroups a compute unit, for which there are no registers, 120.
template <int V, int LPH, bool PAIRS, bool NORM, bool GAINS>
__global__ __launch_bounds__(ROPE_THREADS) void rope_bwd_kernel(const RopeArgs P, const int wgs_q, float* part) {
    typedef typename RopeVec<V>::type Vec;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool is_q = (int)blockIdx.x < wgs_q;
    const int H = is_q ? P.Hq : P.Hkv, at_once = rope_heads_at_once(LPH, H), tokens = 64 / LPH / at_once;
    const int first = (int)blockIdx.x - (is_q ? 0 : wgs_q), wgs = is_q ? wgs_q : (int)gridDim.x - wgs_q;
    const RopeIn G = is_q ? P.gq : P.gk, X = is_q ? P.q : P.k;
    const RopeOut O = is_q ? P.dq : P.dk;
    const bf16_t* gain = is_q ? P.gain_q : P.gain_k;
    RopeLane<V, LPH, PAIRS> L(lane, P.D, P.rot);
    L.frequencies(P);
    Vec gains[2] = {};
    if (NORM && gain != nullptr) {
#pragma unroll
        for (int j = 0; j < 2; ++j) gains[j] = rope_slot<V>(gain, L.col[j], L.has[j]);
    }
    // a unit: the heads that a wavefront works on at once
    const int per_token = (H + at_once - 1) / at_once, my_token = lane / (LPH * at_once), my_head = lane / LPH % at_once;
    const int64_t units = ((int64_t)P.T + tokens - 1) / tokens * per_token;
    struct Unit {
        int t, head;                                     // head < 0: none
        Vec g[2], x[2];
        typename RopeLane<V, LPH, PAIRS>::Place at;
    };
    auto load = [&](int64_t unit, Unit& n) {
        const int64_t tg = unit / per_token, t = tg * tokens + my_token;
        const int h = (int)(unit - tg * per_token) * at_once + my_head;
        const bool ok = t < P.T && h < H;
        n.t = ok ? (int)t : 0;
        n.head = ok ? h : -1;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            // past the last token or head: the first one's, unused
            n.g[j] = rope_slot<V>(G.p + (int64_t)n.t * G.tok + (ok ? h : 0) * G.head, L.col[j], L.has[j]);
            if constexpr (NORM) n.x[j] = rope_slot<V>(X.p + (int64_t)n.t * X.tok + (ok ? h : 0) * X.head, L.col[j], L.has[j]);
        }
        n.at = L.place(P, n.t);
    };
    float sum[2 * V] = {};
    const int64_t step = (int64_t)wgs * ROPE_WAVES;
    const int64_t begin = (int64_t)first * ROPE_WAVES + wave;
    Unit next{};
    for (int64_t unit = begin; unit < units + step; unit += step) {
        const Unit n = next;
        if (unit < units) load(unit, next);
        if (unit == begin) continue;                     // one copy of the loads: code that is run once comes from memory a line at a time
        float cs[V], sn[V], a[V], b[V];
        L.angles(n.at, cs, sn);
        rope_unpack<V>(n.g[0], a);
        rope_unpack<V>(n.g[1], b);
        L.rotate(a, b, cs, sn, true);
        if constexpr (NORM) {
            float xa[V], xb[V], ss = 0.0f, dot = 0.0f;
            rope_unpack<V>(n.x[0], xa);
            rope_unpack<V>(n.x[1], xb);
#pragma unroll
            for (int j = 0; j < V; ++j) ss = fmaf(xa[j], xa[j], fmaf(xb[j], xb[j], ss));
            const float r = rsqrtf(head_sum<LPH>(ss) * P.inv_D + P.eps);
            if (GAINS && n.head >= 0) {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    sum[j] = fmaf(a[j], xa[j] * r, sum[j]);
                    sum[V + j] = fmaf(b[j], xb[j] * r, sum[V + j]);
                }
            }
            if (gain != nullptr) {
                float ga[V], gb[V];
                rope_unpack<V>(gains[0], ga);
                rope_unpack<V>(gains[1], gb);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    a[j] *= ga[j];
                    b[j] *= gb[j];
                }
            }
#pragma unroll
            for (int j = 0; j < V; ++j) dot = fmaf(a[j], xa[j], fmaf(b[j], xb[j], dot));
            const float m = r * r * (head_sum<LPH>(dot) * P.inv_D);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                a[j] = r * (a[j] - xa[j] * m);
                b[j] = r * (b[j] - xb[j] * m);
            }
        }
        if (n.head < 0) continue;
        bf16_t* to = O.p + (int64_t)n.t * O.tok + n.head * O.head;
        if (L.has[0]) *reinterpret_cast<Vec*>(to + L.col[0]) = rope_pack<V>(a);
        if (L.has[1]) *reinterpret_cast<Vec*>(to + L.col[1]) = rope_pack<V>(b);
    }
    if constexpr (GAINS) {
        __shared__ f32x4 lds[2 * V / 4][ROPE_THREADS];
#pragma unroll
        for (int j = 0; j < 2 * V; j += 4) lds[j / 4][threadIdx.x] = f32x4{sum[j], sum[j + 1], sum[j + 2], sum[j + 3]};
        __syncthreads();
        for (int e = threadIdx.x; e < LPH * 2 * V; e += ROPE_THREADS) {
            const int l = e / (2 * V), j = e % (2 * V);
            const RopeLane<V, LPH, PAIRS> M(l, P.D, P.rot);
            const int col = j < V ? M.col[0] : M.col[1];
            if (col >= P.D) continue;
            float v = 0.0f;
            for (int i = l; i < ROPE_THREADS; i += LPH) v += lds[j / 4][i][j % 4];
            part[(int64_t)blockIdx.x * P.D + col + j % V] = v;
        }
    }
}

__global__ __launch_bounds__(32 * COLSUM_LANES) void rope_gain_grad_kernel(const float* part, int wgs_q, int wgs_k, int D, float* dq, float* dk, int accumulate) {
    const bool is_q = blockIdx.y == 0;
    float* out = is_q ? dq : dk;
    if (out == nullptr) return;
    column_sum<COLSUM_LANES>(is_q ? part : part + (int64_t)wgs_q * D, is_q ? wgs_q : wgs_k, D, out, accumulate);
}

namespace {
// slots of 8 columns where the halves (neighbours: the rotated columns) are whole ones
template <class Launch>
void rope_variant(const RopeArgs& a, Launch&& go) {
    if (a.pairs || a.rot % 16 == 0) {
        if (a.D <= 64) go(std::integral_constant<int, 8>{}, std::integral_constant<int, 4>{});
        else go(std::integral_constant<int, 8>{}, std::integral_constant<int, 8>{});
    } else {
        if (a.D <= 64) go(std::integral_constant<int, 4>{}, std::integral_constant<int, 8>{});
        else go(std::integral_constant<int, 4>{}, std::integral_constant<int, 16>{});
    }
}
int rope_heads(const RopeArgs& a) { return a.Hq + a.Hkv + (a.v.p != nullptr ? a.Hkv : 0); }
struct RopeGrid { int chunks; int64_t units; };
RopeGrid rope_grid(const RopeArgs& a, int lph, int heads, int u) {
    const int at_once = rope_heads_at_once(lph, heads), tokens = 64 / lph / at_once;
    RopeGrid g;
    g.chunks = (heads + at_once * u - 1) / (at_once * u);
    g.units = ((int64_t)a.T + tokens - 1) / tokens * g.chunks;
    return g;
}
constexpr int ROPE_BWD_PER_CU = 3;                       // workgroups, by its registers
}  // namespace

// Heads of a wavefront one after the other: one where that many wavefronts find room on the chip at once, otherwise three (us, 32 / 8 heads of 128 into a cache, one / three:
// 64 tokens 4.5 / 6.3, 616 8.4 / 8.9, 1500 14.7 / 12.7, 2944 22.4 / 18.4, 11776 75.7 / 60.3)
template <class Launch>
static void rope_forward_variant(const RopeArgs& a, int ncu, Launch&& go) {
    rope_variant(a, [&](auto v, auto lph) {
        const RopeGrid one = rope_grid(a, decltype(lph)::value, rope_heads(a), 1);
        if (one.units <= (int64_t)ncu * 32) go(v, lph, std::integral_constant<int, 1>{}, one);
        else go(v, lph, std::integral_constant<int, 3>{}, rope_grid(a, decltype(lph)::value, rope_heads(a), 3));
    });
}

int64_t rope_forward_workgroups(const RopeArgs& a, int ncu) {
    int64_t n = 0;
    rope_forward_variant(a, ncu, [&](auto, auto, auto, const RopeGrid& g) { n = (g.units + ROPE_WAVES - 1) / ROPE_WAVES; });
    return n;
}

hipError_t launch_rope_forward(const RopeArgs& a, int ncu, hipStream_t s) {
    rope_forward_variant(a, ncu, [&](auto v, auto lph, auto u, const RopeGrid& g) {
        constexpr int V = decltype(v)::value, LPH = decltype(lph)::value, U = decltype(u)::value;
        const dim3 grid((uint32_t)((g.units + ROPE_WAVES - 1) / ROPE_WAVES));
        if constexpr (V == 8) {
            if (a.pairs && a.norm) rope_fwd_kernel<V, LPH, U, true, true><<<grid, ROPE_THREADS, 0, s>>>(a, g.chunks);
            else if (a.pairs) rope_fwd_kernel<V, LPH, U, true, false><<<grid, ROPE_THREADS, 0, s>>>(a, g.chunks);
        }
        if (!a.pairs && a.norm) rope_fwd_kernel<V, LPH, U, false, true><<<grid, ROPE_THREADS, 0, s>>>(a, g.chunks);
        else if (!a.pairs) rope_fwd_kernel<V, LPH, U, false, false><<<grid, ROPE_THREADS, 0, s>>>(a, g.chunks);
    });
    return hipGetLastError();
}

// Three workgroups a compute unit, shared out by the heads of q and k, but no more than have heads to work on, `rows` of them a wavefront at once
struct RopeShare { int64_t q, k; };
static RopeShare rope_backward_share(int64_t T, int64_t Hq, int64_t Hkv, int rows, int ncu) {
    auto most = [&](int64_t H) { return (T * H + rows * ROPE_WAVES - 1) / (rows * ROPE_WAVES); };
    const int64_t all = (int64_t)ncu * ROPE_BWD_PER_CU;
    const int64_t k = std::min(most(Hkv), std::max<int64_t>(1, (all * Hkv + (Hq + Hkv) / 2) / (Hq + Hkv)));
    return {std::min(most(Hq), std::max<int64_t>(1, all - k)), k};
}
int64_t rope_backward_workgroups(int64_t T, int64_t Hq, int64_t Hkv, int ncu) {
    const RopeShare w = rope_backward_share(T, Hq, Hkv, 4, ncu);      // 16 lanes a head: as many as there can be
    return w.q + w.k;
}

hipError_t launch_rope_backward(const RopeArgs& a, float* part, float* d_gain_q, float* d_gain_k, int accumulate, int ncu, hipStream_t s) {
    const bool gains = d_gain_q != nullptr || d_gain_k != nullptr;
    RopeShare w{0, 0};
    if (a.T > 0)
        rope_variant(a, [&](auto v, auto lph) {
            constexpr int V = decltype(v)::value, LPH = decltype(lph)::value;
            w = rope_backward_share(a.T, a.Hq, a.Hkv, 64 / LPH, ncu);
            const uint32_t wgs = (uint32_t)(w.q + w.k);
            auto go = [&](auto pairs) {
                constexpr bool PAIRS = decltype(pairs)::value;
                if (gains) rope_bwd_kernel<V, LPH, PAIRS, true, true><<<wgs, ROPE_THREADS, 0, s>>>(a, (int)w.q, part);
                else if (a.norm) rope_bwd_kernel<V, LPH, PAIRS, true, false><<<wgs, ROPE_THREADS, 0, s>>>(a, (int)w.q, part);
                else rope_bwd_kernel<V, LPH, PAIRS, false, false><<<wgs, ROPE_THREADS, 0, s>>>(a, (int)w.q, part);
            };
            if constexpr (V == 8) {
                if (a.pairs) go(std::true_type{});
            }
            if (!a.pairs) go(std::false_type{});
        });
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !gains) return e;
    rope_gain_grad_kernel<<<dim3((uint32_t)(a.D + 31) / 32, 2), 32 * COLSUM_LANES, 0, s>>>(part, (int)w.q, (int)w.k, a.D, d_gain_q, d_gain_k, accumulate);
    return hipGetLastError();
}

}  // namespace skipffn
