// Queries and keys normed per head and turned to their positions in one pass, and the gradient of that.
//
// With h = r x, r = (mean_c x_c^2 + eps)^-1/2 over a head's channels, and z = w h (without a weight z = x):
//   y = m R z on the first `rot` channels, R turning the pair (z_a, z_b) of frequency f by a = f pos, y = z
//   on the others; the pairs are (c, c + rot / 2), or neighbours (2c, 2c + 1).
// Backwards, with g = m R^T dy (g = dy on the channels that are not turned) and u = w g:
//   dx = r (u - h mean_c(u h)),   dw_c = sum over tokens and heads of g_c h_c.
//
// V = 16 / sizeof(T); a thread holds V pairs of a head, both channels of each, as two 16-byte pieces, so that
// the turn needs no other lane: D / 2V lanes make a head, and its sums take log2 of that many exchanges. A
// thread keeps its V angles for all heads of its token. Everything is bound by HBM, each element read once
// and written once; arithmetic and statistics are fp32, angles 64-bit fractions of a turn (rows.cuh).
#include <algorithm>
#include <cstdint>

#include "rows.cuh"
#include "serve.h"

namespace ris {
namespace {

using rows::sincos_turns;
using rows::Vec;

constexpr int kThreads = 256, kBatch = 2;

// The pairs of a thread: lane l of a head's D / 2V.
template <typename T, bool PAIRS>
struct Lane {
    static constexpr int V = Vec<T>::V;
    int at[2];   // first channel of its two pieces
    int f;       // its first frequency
    bool turns;  // whether its channels are among the first `rot`
    __device__ __forceinline__ Lane(int l, int rot)
    {
        const int n = rot / (2 * V);  // lanes that turn
        turns = l < n;
        f = V * l;
        at[0] = PAIRS || !turns ? 2 * V * l : V * l;
        at[1] = PAIRS || !turns ? at[0] + V : at[0] + rot / 2;
    }
    // element e of the thread's 2 V as (pair, which): of its first channels for i = 0, of its second for 1
    static __device__ __forceinline__ float get(const Vec<T> (&p)[2], int i, int e)
    {
        return PAIRS ? p[(2 * e + i) / V][(2 * e + i) % V] : p[i][e];
    }
    static __device__ __forceinline__ void put(T *row, const int (&at)[2], const float (&a)[V], const float (&b)[V])
    {
        float p[2][V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            if constexpr (PAIRS) {
                p[2 * e / V][2 * e % V] = a[e];
                p[(2 * e + 1) / V][(2 * e + 1) % V] = b[e];
            } else {
                p[0][e] = a[e];
                p[1][e] = b[e];
            }
        }
        Vec<T>::store(row + at[0], p[0]);
        Vec<T>::store(row + at[1], p[1]);
    }
    static __device__ __forceinline__ void load(Vec<T> (&p)[2], const T *row, const int (&at)[2])
    {
        p[0].load(row + at[0]);
        p[1].load(row + at[1]);
    }
};

// x summed over the n lanes of a head (n a power of two, aligned)
__device__ __forceinline__ float head_sum(float x, int n)
{
    for (int o = n >> 1; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
    return x;
}

template <typename T, bool PAIRS, int D>
__global__ void __launch_bounds__(kThreads, 2) k_norm_rope(const __grid_constant__ NormRopeArgs a)
{
    using L = Lane<T, PAIRS>;
    constexpr int V = L::V, LANES = D / (2 * V), TOKENS = kThreads / LANES;
    const int l = threadIdx.x % LANES;
    const L lane(l, a.rot);
    const int64_t p = (int64_t)blockIdx.x * TOKENS + threadIdx.x / LANES;
    const bool there = p < a.n;
    const int64_t row = there ? p : 0;  // (lanes past the last token take part in the exchanges)
    after_last();
    // heads h0 .. h1 - 1 of q and k, one after another
    const int heads = a.heads[0] + a.heads[1];
    const int h0 = (int)((int64_t)heads * blockIdx.y / gridDim.y), h1 = (int)((int64_t)heads * (blockIdx.y + 1) / gridDim.y);
    auto in = [&](int h) {
        const int w = h >= a.heads[0];
        return reinterpret_cast<const T *>(a.x[w]) + row * a.x_stride[w] + (h - w * a.heads[0]) * D;
    };
    // kBatch heads' loads ahead of what is stored before them in time (which the compiler may not reorder:
    // they may be in place), the first ahead of the sines and cosines
    Vec<T> next[kBatch][2];
    auto load = [&](int h) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
            if (h + i < h1) L::load(next[i], in(h + i), lane.at);
    };
    load(h0);
    float cs[V], sn[V];
    if (lane.turns) {
        const int32_t pos = a.pos[row];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            sincos_turns(pos, a.turn[lane.f + e], &sn[e], &cs[e]);
            cs[e] *= a.mscale;
            sn[e] *= a.mscale;
        }
    }
    float wa[V], wb[V];
    const void *weight = nullptr;
    bool first = true;
    for (int h = h0; h < h1; h += kBatch) {
        Vec<T> x[kBatch][2];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) x[i][0] = next[i][0], x[i][1] = next[i][1];
        load(h + kBatch);
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            if (h + i >= h1) break;
            const int w = h + i >= a.heads[0];
            if (first || (w == 1 && h + i == a.heads[0])) {
                first = false;
                weight = a.weight[w];
                Vec<T> p[2];
                if (weight != nullptr) L::load(p, reinterpret_cast<const T *>(weight), lane.at);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    wa[e] = weight != nullptr ? L::get(p, 0, e) : 1.f;
                    wb[e] = weight != nullptr ? L::get(p, 1, e) : 1.f;
                }
            }
            float r = 1.f;
            if (weight != nullptr) {  // (the same for all threads)
                float s = 0.f;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float u = L::get(x[i], 0, e), v = L::get(x[i], 1, e);
                    s = fmaf(u, u, fmaf(v, v, s));
                }
                r = rsqrtf(fmaf(head_sum(s, LANES), 1.f / D, a.eps));
            }
            float ya[V], yb[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float u = L::get(x[i], 0, e) * r * wa[e], v = L::get(x[i], 1, e) * r * wb[e];
                ya[e] = lane.turns ? fmaf(u, cs[e], -(v * sn[e])) : u;
                yb[e] = lane.turns ? fmaf(v, cs[e], u * sn[e]) : v;
            }
            if (there)
                L::put(reinterpret_cast<T *>(a.y[w]) + row * a.y_stride[w] + (h + i - w * a.heads[0]) * D, lane.at, ya, yb);
        }
    }
}

// The gradient. A CTA belongs to q or to k (the sums of a weight's gradient stay in its threads' registers)
// and takes every step-th group of tokens of it; what its threads summed is added up in a fixed order here
// and over the CTAs in k_weight_sums, so that no result depends on the order in which they run.
template <typename T, bool PAIRS, int D>
__global__ void __launch_bounds__(kThreads, 2) k_norm_rope_backward(const __grid_constant__ NormRopeArgs a)
{
    using L = Lane<T, PAIRS>;
    constexpr int V = L::V, LANES = D / (2 * V), TOKENS = kThreads / LANES;
    __shared__ float part[TOKENS][D + 1];
    const int l = threadIdx.x % LANES, group = threadIdx.x / LANES;
    const L lane(l, a.rot);
    const int w = (int)blockIdx.x >= a.ctas[0], cta = blockIdx.x - (w ? a.ctas[0] : 0), heads = a.heads[w];
    after_last();
    const void *const weight = a.weight[w];
    float wa[V], wb[V], ga[V], gb[V];
    {
        Vec<T> p[2];
        if (weight != nullptr) L::load(p, reinterpret_cast<const T *>(weight), lane.at);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            wa[e] = weight != nullptr ? L::get(p, 0, e) : 1.f;
            wb[e] = weight != nullptr ? L::get(p, 1, e) : 1.f;
            ga[e] = gb[e] = 0.f;
        }
    }
    for (int64_t p0 = (int64_t)cta * TOKENS; p0 < a.n; p0 += (int64_t)a.ctas[w] * TOKENS) {
        const bool there = p0 + group < a.n;
        const int64_t row = there ? p0 + group : 0;
        const T *const xr = reinterpret_cast<const T *>(a.x[w]) + row * a.x_stride[w], *const dr = reinterpret_cast<const T *>(a.dy[w]) + row * a.dy_stride[w];
        T *const yr = reinterpret_cast<T *>(a.y[w]) + row * a.y_stride[w];
        Vec<T> xn[2], dn[2];
        L::load(dn, dr, lane.at);
        if (weight != nullptr) L::load(xn, xr, lane.at);
        float cs[V], sn[V];
        if (lane.turns) {
            const int32_t pos = a.pos[row];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                sincos_turns(pos, a.turn[lane.f + e], &sn[e], &cs[e]);
                cs[e] *= a.mscale;
                sn[e] *= a.mscale;
            }
        }
        for (int h = 0; h < heads; ++h) {
            const Vec<T> x[2] = {xn[0], xn[1]}, d[2] = {dn[0], dn[1]};
            if (h + 1 < heads) {  // (ahead of the stores, which may be in place)
                L::load(dn, dr + (h + 1) * D, lane.at);
                if (weight != nullptr) L::load(xn, xr + (h + 1) * D, lane.at);
            }
            float ua[V], ub[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float u = L::get(d, 0, e), v = L::get(d, 1, e);
                ua[e] = lane.turns ? fmaf(u, cs[e], v * sn[e]) : u;
                ub[e] = lane.turns ? fmaf(v, cs[e], -(u * sn[e])) : v;
            }
            if (weight != nullptr) {  // (the same for all threads)
                float s = 0.f, t = 0.f;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float u = L::get(x, 0, e), v = L::get(x, 1, e);
                    s = fmaf(u, u, fmaf(v, v, s));
                    t = fmaf(ua[e] * wa[e], u, fmaf(ub[e] * wb[e], v, t));
                }
                const float r = rsqrtf(fmaf(head_sum(s, LANES), 1.f / D, a.eps));
                const float mean = head_sum(t, LANES) * r * (1.f / D);  // of u h
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float hu = L::get(x, 0, e) * r, hv = L::get(x, 1, e) * r;
                    if (there) {
                        ga[e] = fmaf(ua[e], hu, ga[e]);
                        gb[e] = fmaf(ub[e], hv, gb[e]);
                    }
                    ua[e] = r * fmaf(-mean, hu, ua[e] * wa[e]);
                    ub[e] = r * fmaf(-mean, hv, ub[e] * wb[e]);
                }
            }
            if (there) L::put(yr + h * D, lane.at, ua, ub);
        }
    }
    if (weight == nullptr) return;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const int ca = PAIRS ? 2 * e : e, cb = PAIRS ? 2 * e + 1 : V + e;
        part[group][lane.at[ca / V] + ca % V] = ga[e];
        part[group][lane.at[cb / V] + cb % V] = gb[e];
    }
    __syncthreads();
    for (int c = threadIdx.x; c < D; c += kThreads) {
        float s = 0.f;
        for (int i = 0; i < TOKENS; ++i) s += part[i][c];
        a.part[(int64_t)blockIdx.x * D + c] = s;
    }
}

// dw of q (block 0) and k (block 1): the CTAs' sums, in 64 bits.
template <int D>
__global__ void __launch_bounds__(1024) k_weight_sums(const float *part, int ctas_q, int ctas_k, float *gq, float *gk)
{
    constexpr int S = 1024 / D;
    __shared__ double sums[S][D];
    const int w = blockIdx.x, c = threadIdx.x % D, i0 = threadIdx.x / D, n = w ? ctas_k : ctas_q;
    float *const out = w ? gk : gq;
    after_last();
    if (out == nullptr) return;
    part += (int64_t)(w ? ctas_q : 0) * D + c;
    double s = 0.0;
#pragma unroll 8
    for (int i = i0; i < n; i += S) s += (double)part[(int64_t)i * D];
    sums[i0][c] = s;
    __syncthreads();
    if (i0 != 0) return;
    for (int i = 1; i < S; ++i) s += sums[i][c];
    out[c] = (float)s;
}

template <typename T, bool PAIRS, int D>
cudaError_t forward(const NormRopeArgs &a, cudaStream_t s)
{
    constexpr int TOKENS = kThreads / (D / (2 * Vec<T>::V));
    const int64_t blocks = (a.n + TOKENS - 1) / TOKENS;
    const int heads = a.heads[0] + a.heads[1];
    // two CTAs per SM before a slice holds every head
    const int slices = (int)std::min<int64_t>(heads, std::max<int64_t>(1, 304 / blocks));
    return launch_chained(k_norm_rope<T, PAIRS, D>, dim3((unsigned)blocks, (unsigned)slices), dim3(kThreads), 0, s, a);
}

template <typename T, bool PAIRS, int D>
cudaError_t backward(const NormRopeArgs &a, float *gq, float *gk, cudaStream_t s)
{
    if (a.n > 0) {
        const cudaError_t e = launch_chained(k_norm_rope_backward<T, PAIRS, D>, dim3((unsigned)(a.ctas[0] + a.ctas[1])), dim3(kThreads), 0, s, a);
        if (e != cudaSuccess) return e;
    }
    if (gq == nullptr && gk == nullptr) return cudaSuccess;
    const int n0 = a.n > 0 ? a.ctas[0] : 0, n1 = a.n > 0 ? a.ctas[1] : 0;
    return launch_chained(k_weight_sums<D>, dim3(2), dim3(1024), 0, s, static_cast<const float *>(a.part), n0, n1, gq, gk);
}

}  // namespace

// CTAs of the gradient's kernel for q and for k: two to an SM in all, shared out by heads, and no more than
// there are groups of tokens.
void norm_rope_ctas(int dtype, int D, int64_t n, const int32_t (&heads)[2], int32_t (&ctas)[2])
{
    const int tokens = kThreads / (D / (2 * (dtype == RIS_F32 ? 4 : 8)));
    const int64_t groups = std::max<int64_t>(1, (n + tokens - 1) / tokens);
    const int all = heads[0] + heads[1];
    for (int w = 0; w < 2; ++w)
        ctas[w] = heads[w] == 0 ? 0 : (int32_t)std::min<int64_t>(groups, std::max<int64_t>(1, (304LL * heads[w] + all / 2) / all));
}

cudaError_t launch_norm_rope(const NormRopeArgs &a, int dtype, int D, bool pairs, cudaStream_t s)
{
    if (dtype == RIS_F32) {
        if (D == 128) return pairs ? forward<float, true, 128>(a, s) : forward<float, false, 128>(a, s);
        return pairs ? forward<float, true, 64>(a, s) : forward<float, false, 64>(a, s);
    }
    if (D == 128) return pairs ? forward<__nv_bfloat16, true, 128>(a, s) : forward<__nv_bfloat16, false, 128>(a, s);
    return pairs ? forward<__nv_bfloat16, true, 64>(a, s) : forward<__nv_bfloat16, false, 64>(a, s);
}

cudaError_t launch_norm_rope_backward(const NormRopeArgs &a, int dtype, int D, bool pairs, float *gq, float *gk, cudaStream_t s)
{
    if (dtype == RIS_F32) {
        if (D == 128) return pairs ? backward<float, true, 128>(a, gq, gk, s) : backward<float, false, 128>(a, gq, gk, s);
        return pairs ? backward<float, true, 64>(a, gq, gk, s) : backward<float, false, 64>(a, gq, gk, s);
    }
    if (D == 128) return pairs ? backward<__nv_bfloat16, true, 128>(a, gq, gk, s) : backward<__nv_bfloat16, false, 128>(a, gq, gk, s);
    return pairs ? backward<__nv_bfloat16, true, 64>(a, gq, gk, s) : backward<__nv_bfloat16, false, 64>(a, gq, gk, s);
}

}  // namespace ris
