// Rotary positions given per token, on one axis or on several (time, height, width), of q and k in
// one launch, out of the rows of a fused projection or in place.
//
// y_c = m (x_c cos a - x_{c+D/2} sin a), y_{c+D/2} = m (x_{c+D/2} cos a + x_c sin a) with a = f_c
// pos[axis(c)][token]; the transposed rotation (inverse) turns by -a and is the gradient's.
//
// One thread takes V = 16 / sizeof(T) frequencies of a token (16-byte accesses of both halves of a head),
// forms their sines and cosines once and turns every head of its slice. Angles are 64-bit fixed-point
// fractions of a turn, as in the layer calls' rotation: exact at any int32 position, where a product in
// fp32 is off by 1e-3 at position 30,000. Bound by HBM: each element read once and written once; the sines
// and cosines (about 40 instructions each) are shared by the heads. The heads are sliced over CTAs only
// where the tokens alone leave SMs without work, since every slice repeats the sines and cosines. 30,011
// tokens of 12 and 2 heads of 128 in bf16 on three axes take 37.7 us, 5.7 TB/s of the 6.8 that a copy
// reaches; 24 tokens are a launch's latency.
#include <algorithm>
#include <cstdint>

#include "rows.cuh"
#include "serve.h"

namespace ris {
namespace {

using rows::sincos_turns;
using rows::Vec;

constexpr int kThreads = 256, kBatch = 2;

template <typename T>
__global__ void __launch_bounds__(kThreads, 4) k_rope_axes(const RopeAxesArgs a)
{
    constexpr int V = Vec<T>::V;
    const int half = a.D >> 1, c = V * threadIdx.x;  // blockDim.x == half / V
    const int64_t p = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    after_last();
    if (p >= a.n) return;
    // heads h0 .. h1 - 1 of q and k, one after another
    const int heads = a.heads[0] + a.heads[1];
    const int h0 = (int)((int64_t)heads * blockIdx.y / gridDim.y), h1 = (int)((int64_t)heads * (blockIdx.y + 1) / gridDim.y);
    auto of = [&](int h, bool out) -> T * {
        const int w = h >= a.heads[0];
        const int64_t at = p * (out ? (int64_t)a.heads[w] * a.D : a.stride[w]) + (h - w * a.heads[0]) * a.D + c;
        return (out ? reinterpret_cast<T *>(a.y[w]) : reinterpret_cast<T *>(const_cast<void *>(a.x[w]))) + at;
    };
    // kBatch heads' loads ahead of what is stored before them in time (which the compiler may not reorder:
    // they may be in place), the first ahead of the sines and cosines
    Vec<T> u[kBatch], v[kBatch];
    auto load = [&](int h) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
            if (h + i < h1) {
                const T *x = of(h + i, false);
                u[i].load(x);
                v[i].load(x + half);
            }
    };
    load(h0);
    float cs[V], sn[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        sincos_turns(a.pos[(int64_t)a.axis[c + e] * a.n + p], a.turn[c + e], &sn[e], &cs[e]);
        cs[e] *= a.mscale;
        sn[e] *= a.inverse ? -a.mscale : a.mscale;
    }
    for (int h = h0; h < h1; h += kBatch) {
        Vec<T> s[kBatch], t[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            s[i] = u[i];
            t[i] = v[i];
        }
        load(h + kBatch);
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
            if (h + i < h1) {
                float x[V], y[V];
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    x[e] = fmaf(s[i][e], cs[e], -(t[i][e] * sn[e]));
                    y[e] = fmaf(t[i][e], cs[e], s[i][e] * sn[e]);
                }
                T *out = of(h + i, true);
                Vec<T>::store(out, x);
                Vec<T>::store(out + half, y);
            }
    }
}

template <typename T>
cudaError_t launch(const RopeAxesArgs &a, cudaStream_t s)
{
    const int x = a.D / 2 / Vec<T>::V, tokens = kThreads / x;
    const int64_t blocks = (a.n + tokens - 1) / tokens;
    const int heads = a.heads[0] + a.heads[1];
    // two CTAs per SM before a slice holds every head
    const int slices = (int)std::min<int64_t>(heads, std::max<int64_t>(1, 304 / blocks));
    return launch_chained(k_rope_axes<T>, dim3((unsigned)blocks, (unsigned)slices), dim3(x, tokens), 0, s, a);
}

}  // namespace

cudaError_t launch_rope_axes(const RopeAxesArgs &a, int dtype, cudaStream_t s)
{
    return dtype == RIS_F32 ? launch<float>(a, s) : launch<__nv_bfloat16>(a, s);
}

}  // namespace ris
