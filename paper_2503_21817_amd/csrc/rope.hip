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
// [-1, 1] half turns there, sine and cosine in 32.
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
    // cosine and sine of the lane's frequencies u V + i for a token
    __device__ __forceinline__ void angles(const RopeArgs& P, int t, float (&cs)[V], float (&sn)[V]) const {
        int32_t pos[ROPE_MAX_AXES];
#pragma unroll
        for (int a = 0; a < ROPE_MAX_AXES; ++a) pos[a] = a < P.n_axes ? P.pos[(int64_t)a * P.T + t] : 0;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int j = u * V + i;
            const bool in = j < P.rot / 2;
            const int axis = in && P.n_axes > 1 ? P.axis[in ? j : 0] : 0;
            int32_t p = pos[0];
#pragma unroll
            for (int a = 1; a < ROPE_MAX_AXES; ++a) p = axis == a ? pos[a] : p;
            const double x = (double)p * (double)(in ? P.inv_freq[j] : 0.0f) * 0.31830988618379067154;       // in half turns
            const float f = (float)(x - 2.0 * rint(x * 0.5));
            sincospif(f, &sn[i], &cs[i]);
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

template <int LPH>
__device__ __forceinline__ float head_sum(float v) {
#pragma unroll
    for (int off = LPH / 2; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    return v;
}

// Heads that a wavefront has at a time, and tokens beside one another: powers of two whose product with LPH is 64
__host__ __device__ inline int rope_heads_at_once(int lph, int heads) {
    int n = 1;
    while (n * 2 * lph <= 64 && n < heads) n *= 2;
    return n;
}

// A wavefront has U times as many heads of its tokens as it works on at once; all of their loads are asked for first
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
    const RopeLane<V, LPH, PAIRS> L(lane, P.D, P.rot);
    const int64_t row = P.row != nullptr ? (int64_t)P.row[t] : t;
    const bool stored = row >= 0 && row < P.rows_out;    // of k and v
    int head[U];
    bf16_t* to[U];
    Vec x[U][2];
#pragma unroll
    for (int i = 0; i < U; ++i) {
        head[i] = (chunk * U + i) * at_once + lane / LPH % at_once;
        const bf16_t* from = nullptr;
        to[i] = nullptr;
        if (head[i] < P.Hq) {
            from = P.q.p + (int64_t)t * P.q.tok + head[i] * P.q.head;
            to[i] = P.q_out.p + (int64_t)t * P.q_out.tok + head[i] * P.q_out.head;
        } else if (head[i] < heads && stored) {
            const int h = head[i] - P.Hq;
            const bool is_k = h < P.Hkv;
            from = is_k ? P.k.p + (int64_t)t * P.k.tok + h * P.k.head : P.v.p + (int64_t)t * P.v.tok + (h - P.Hkv) * P.v.head;
            to[i] = is_k ? P.k_out.p + row * P.k_out.tok + h * P.k_out.head : P.v_out.p + row * P.v_out.tok + (h - P.Hkv) * P.v_out.head;
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) x[i][j] = from != nullptr && L.has[j] ? *reinterpret_cast<const Vec*>(from + L.col[j]) : Vec{};
    }
    float cs[V], sn[V];
    L.angles(P, t, cs, sn);
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
                const float r = rsqrtf(head_sum<LPH>(ss) / (float)P.D + P.eps);
                const bf16_t* gain = head[i] < P.Hq ? P.gain_q : P.gain_k;
                float ga[V], gb[V];
                if (gain != nullptr) {
                    rope_unpack<V>(L.has[0] ? *reinterpret_cast<const Vec*>(gain + L.col[0]) : Vec{}, ga);
                    rope_unpack<V>(L.has[1] ? *reinterpret_cast<const Vec*>(gain + L.col[1]) : Vec{}, gb);
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

// Workgroups go on through the tokens; with gain gradients every lane keeps the sums of its columns, joined over the workgroup at the end:
// part [q or k][workgroup][D]
template <int V, int LPH, int U, bool PAIRS, bool NORM, bool GAINS>
__global__ __launch_bounds__(ROPE_THREADS) void rope_bwd_kernel(const RopeArgs P, const int chunks, const int64_t units, float* part) {
    typedef typename RopeVec<V>::type Vec;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int heads = P.Hq + P.Hkv, at_once = rope_heads_at_once(LPH, heads), tokens = 64 / LPH / at_once;
    const RopeLane<V, LPH, PAIRS> L(lane, P.D, P.rot);
    float sum[GAINS ? 2 : 1][2 * V] = {};
    for (int64_t unit = (int64_t)blockIdx.x * ROPE_WAVES + wave; unit < units; unit += (int64_t)gridDim.x * ROPE_WAVES) {
        const int64_t group = unit / chunks;
        const int chunk = (int)(unit - group * chunks);
        const int64_t t64 = group * tokens + lane / (LPH * at_once);
        const bool in = t64 < P.T;
        const int t = in ? (int)t64 : 0;
        int head[U];
        Vec g[U][2], x[U][2];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            head[i] = (chunk * U + i) * at_once + lane / LPH % at_once;
            const bool ok = in && head[i] < heads, is_q = head[i] < P.Hq;
            const int h = is_q ? head[i] : head[i] - P.Hq;
            const RopeIn &G = is_q ? P.gq : P.gk, &X = is_q ? P.q : P.k;
            if (!ok) head[i] = heads;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                g[i][j] = ok && L.has[j] ? *reinterpret_cast<const Vec*>(G.p + (int64_t)t * G.tok + h * G.head + L.col[j]) : Vec{};
                if constexpr (NORM) x[i][j] = ok && L.has[j] ? *reinterpret_cast<const Vec*>(X.p + (int64_t)t * X.tok + h * X.head + L.col[j]) : Vec{};
            }
        }
        float cs[V], sn[V];
        L.angles(P, t, cs, sn);
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const bool is_q = head[i] < P.Hq;
            float a[V], b[V];
            rope_unpack<V>(g[i][0], a);
            rope_unpack<V>(g[i][1], b);
            L.rotate(a, b, cs, sn, true);
            if constexpr (NORM) {
                float xa[V], xb[V], ss = 0.0f, dot = 0.0f;
                rope_unpack<V>(x[i][0], xa);
                rope_unpack<V>(x[i][1], xb);
#pragma unroll
                for (int j = 0; j < V; ++j) ss = fmaf(xa[j], xa[j], fmaf(xb[j], xb[j], ss));
                const float r = rsqrtf(head_sum<LPH>(ss) / (float)P.D + P.eps);
                const bf16_t* gain = is_q ? P.gain_q : P.gain_k;
                if constexpr (GAINS) {
                    const bool ok = head[i] < heads;
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const float da = ok ? a[j] * (xa[j] * r) : 0.0f, db = ok ? b[j] * (xb[j] * r) : 0.0f;
                        sum[0][j] += is_q ? da : 0.0f;
                        sum[0][V + j] += is_q ? db : 0.0f;
                        sum[1][j] += is_q ? 0.0f : da;
                        sum[1][V + j] += is_q ? 0.0f : db;
                    }
                }
                if (gain != nullptr) {
                    float ga[V], gb[V];
                    rope_unpack<V>(L.has[0] ? *reinterpret_cast<const Vec*>(gain + L.col[0]) : Vec{}, ga);
                    rope_unpack<V>(L.has[1] ? *reinterpret_cast<const Vec*>(gain + L.col[1]) : Vec{}, gb);
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        a[j] *= ga[j];
                        b[j] *= gb[j];
                    }
                }
#pragma unroll
                for (int j = 0; j < V; ++j) dot = fmaf(a[j], xa[j], fmaf(b[j], xb[j], dot));
                const float m = r * r * (head_sum<LPH>(dot) / (float)P.D);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    a[j] = r * (a[j] - xa[j] * m);
                    b[j] = r * (b[j] - xb[j] * m);
                }
            }
            if (head[i] >= heads) continue;
            const RopeOut& O = is_q ? P.dq : P.dk;
            bf16_t* to = O.p + (int64_t)t * O.tok + (is_q ? head[i] : head[i] - P.Hq) * O.head;
            if (L.has[0]) *reinterpret_cast<Vec*>(to + L.col[0]) = rope_pack<V>(a);
            if (L.has[1]) *reinterpret_cast<Vec*>(to + L.col[1]) = rope_pack<V>(b);
        }
    }
    if constexpr (GAINS) {
        __shared__ float lds[ROPE_WAVES][2][LPH * 2 * V];
#pragma unroll
        for (int z = 0; z < 2; ++z)
#pragma unroll
            for (int j = 0; j < 2 * V; ++j) {
                float v = sum[z][j];
#pragma unroll
                for (int off = LPH; off < 64; off *= 2) v += __shfl_xor(v, off, 64);
                if (lane < LPH) lds[wave][z][lane * 2 * V + j] = v;
            }
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * LPH * 2 * V; i += ROPE_THREADS) {
            const int z = i / (LPH * 2 * V), e = i % (LPH * 2 * V), j = e % (2 * V);
            const RopeLane<V, LPH, PAIRS> M(e / (2 * V), P.D, P.rot);
            const int s = j / V;
            if (!M.has[s]) continue;
            float v = 0.0f;
#pragma unroll
            for (int w = 0; w < ROPE_WAVES; ++w) v += lds[w][z][e];
            part[((int64_t)z * gridDim.x + blockIdx.x) * P.D + M.col[s] + j % V] = v;
        }
    }
}

__global__ __launch_bounds__(32 * COLSUM_LANES) void rope_gain_grad_kernel(const float* part, int rows, int D, float* dq, float* dk, int accumulate) {
    float* out = blockIdx.y == 0 ? dq : dk;
    if (out == nullptr) return;
    column_sum<COLSUM_LANES>(part + (int64_t)blockIdx.y * rows * D, rows, D, out, accumulate);
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
constexpr int ROPE_FWD_U = 2, ROPE_BWD_U = 2;
}  // namespace

int64_t rope_forward_workgroups(const RopeArgs& a) {
    int64_t n = 0;
    rope_variant(a, [&](auto, auto lph) {
        n = (rope_grid(a, decltype(lph)::value, rope_heads(a), ROPE_FWD_U).units + ROPE_WAVES - 1) / ROPE_WAVES;
    });
    return n;
}

hipError_t launch_rope_forward(const RopeArgs& a, hipStream_t s) {
    rope_variant(a, [&](auto v, auto lph) {
        constexpr int V = decltype(v)::value, LPH = decltype(lph)::value;
        const RopeGrid g = rope_grid(a, LPH, rope_heads(a), ROPE_FWD_U);
        const dim3 grid((uint32_t)((g.units + ROPE_WAVES - 1) / ROPE_WAVES));
        if constexpr (V == 8) {
            if (a.pairs && a.norm) rope_fwd_kernel<V, LPH, ROPE_FWD_U, true, true><<<grid, ROPE_THREADS, 0, s>>>(a, g.chunks);
            else if (a.pairs) rope_fwd_kernel<V, LPH, ROPE_FWD_U, true, false><<<grid, ROPE_THREADS, 0, s>>>(a, g.chunks);
        }
        if (!a.pairs && a.norm) rope_fwd_kernel<V, LPH, ROPE_FWD_U, false, true><<<grid, ROPE_THREADS, 0, s>>>(a, g.chunks);
        else if (!a.pairs) rope_fwd_kernel<V, LPH, ROPE_FWD_U, false, false><<<grid, ROPE_THREADS, 0, s>>>(a, g.chunks);
    });
    return hipGetLastError();
}

int64_t rope_backward_workgroups(int64_t T, int64_t Hq, int64_t Hkv, int ncu) {
    const int64_t most = (T * (Hq + Hkv) + ROPE_WAVES - 1) / ROPE_WAVES;
    return std::max<int64_t>(1, std::min<int64_t>(most, (int64_t)ncu * 4));
}

hipError_t launch_rope_backward(const RopeArgs& a, float* part, float* d_gain_q, float* d_gain_k, int accumulate, int ncu, hipStream_t s) {
    const bool gains = d_gain_q != nullptr || d_gain_k != nullptr;
    const int64_t most = rope_backward_workgroups(a.T, a.Hq, a.Hkv, ncu);
    uint32_t wgs = 0;
    rope_variant(a, [&](auto v, auto lph) {
        constexpr int V = decltype(v)::value, LPH = decltype(lph)::value;
        const RopeGrid g = rope_grid(a, LPH, a.Hq + a.Hkv, ROPE_BWD_U);
        wgs = (uint32_t)std::min<int64_t>((g.units + ROPE_WAVES - 1) / ROPE_WAVES, most);
        if (wgs == 0) return;
        auto go = [&](auto pairs) {
            constexpr bool PAIRS = decltype(pairs)::value;
            if (gains) rope_bwd_kernel<V, LPH, ROPE_BWD_U, PAIRS, true, true><<<wgs, ROPE_THREADS, 0, s>>>(a, g.chunks, g.units, part);
            else if (a.norm) rope_bwd_kernel<V, LPH, ROPE_BWD_U, PAIRS, true, false><<<wgs, ROPE_THREADS, 0, s>>>(a, g.chunks, g.units, part);
            else rope_bwd_kernel<V, LPH, ROPE_BWD_U, PAIRS, false, false><<<wgs, ROPE_THREADS, 0, s>>>(a, g.chunks, g.units, part);
        };
        if constexpr (V == 8) {
            if (a.pairs) go(std::true_type{});
        }
        if (!a.pairs) go(std::false_type{});
    });
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !gains) return e;
    rope_gain_grad_kernel<<<dim3((uint32_t)(a.D + 31) / 32, 2), 32 * COLSUM_LANES, 0, s>>>(part, (int)wgs, a.D, d_gain_q, d_gain_k, accumulate);
    return hipGetLastError();
}

}  // namespace skipffn
