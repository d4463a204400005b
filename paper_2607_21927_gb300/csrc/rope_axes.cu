// Rotary positions given per token, on one axis or on several (time, height, width), of q and k in
// one launch, out of the rows of a fused projection or in place.
//
// y_c = m (x_c cos a - x_{c+D/2} sin a), y_{c+D/2} = m (x_{c+D/2} cos a + x_c sin a) with a = f_c
// pos[axis(c)][token]; the transposed rotation (inverse) turns by -a and is the gradient's.
//
// One thread takes V = 16 / sizeof(T) frequencies of a token (16-byte accesses of both halves of a
// head), forms their sines and cosines once and turns every head of its slice. Angles are 64-bit fixed-point fractions of a
// turn, as in the layer calls' rotation: exact at any int32 position, where a product in fp32 is off by
// 1e-3 at position 30,000. Bound by HBM: each element read once and written once; the sines and cosines
// (about 40 instructions each) are shared by the heads. The heads are sliced over CTAs only where the
// tokens alone leave SMs without work, since every slice repeats the sines and cosines.
#include <cuda_bf16.h>

#include <algorithm>
#include <cstdint>

#include "serve.h"

namespace ris {
namespace {

constexpr int kThreads = 256, kBatch = 4;

template <typename T>
struct Vec;
template <>
struct Vec<float> {
    static constexpr int V = 4;
    static __device__ __forceinline__ void load(const float *p, float *x)
    {
        const float4 v = *reinterpret_cast<const float4 *>(p);
        x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
    }
    static __device__ __forceinline__ void store(float *p, const float *x)
    {
        *reinterpret_cast<float4 *>(p) = make_float4(x[0], x[1], x[2], x[3]);
    }
};
template <>
struct Vec<__nv_bfloat16> {
    static constexpr int V = 8;
    static __device__ __forceinline__ void load(const __nv_bfloat16 *p, float *x)
    {
        const uint4 v = *reinterpret_cast<const uint4 *>(p);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[2 * e] = __uint_as_float(w[e] << 16);
            x[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
        }
    }
    static __device__ __forceinline__ void store(__nv_bfloat16 *p, const float *x)
    {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * e], x[2 * e + 1]);
            w[e] = *reinterpret_cast<const uint32_t *>(&b);
        }
        *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    }
};

// sin and cos of position p (of either sign) times a frequency given as a fraction of a turn in 2^-64:
// the low 64 bits of the product are the fraction of the turn, signed; 2 pi in fp32, the fraction's
// top 24 bits exact and the rest as a correction.
__device__ __forceinline__ void sincos_turns(int32_t p, uint64_t turn, float *sn, float *cs)
{
    const int64_t frac = (int64_t)(turn * (uint64_t)(int64_t)p);
    const float top = (float)(int32_t)(frac >> 40), rest = (float)(uint32_t)(frac >> 8);
    constexpr float A = 0x1.921fb6p-22f, A_LO = -0x1.777a5cp-47f, B = 0x1.921fb6p-54f;  // 2 pi 2^-24 (hi, lo), 2 pi 2^-56
    sincosf(fmaf(top, A, fmaf(top, A_LO, rest * B)), sn, cs);
}

template <typename T>
__global__ void __launch_bounds__(kThreads) k_rope_axes(const RopeAxesArgs a)
{
    constexpr int V = Vec<T>::V;
    const int half = a.D >> 1, c = V * threadIdx.x;  // blockDim.x == half / V
    const int64_t p = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    if (p >= a.n) return;
    const int heads = a.heads[0] + a.heads[1];
    const int h0 = (int)((int64_t)heads * blockIdx.y / gridDim.y), h1 = (int)((int64_t)heads * (blockIdx.y + 1) / gridDim.y);
    float cs[V], sn[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        sincos_turns(a.pos[(int64_t)a.axis[c + e] * a.n + p], a.turn[c + e], &sn[e], &cs[e]);
        cs[e] *= a.mscale;
        sn[e] *= a.inverse ? -a.mscale : a.mscale;
    }
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        const int first = w == 0 ? 0 : a.heads[0], n = a.heads[w];
        const T *x = reinterpret_cast<const T *>(a.x[w]) + p * a.stride[w] + c;
        T *y = reinterpret_cast<T *>(a.y[w]) + p * (int64_t)n * a.D + c;
        // kBatch heads' loads ahead of their stores (which the compiler may not pass: they may be in place)
        const int end = min(h1 - first, n);
        for (int h = max(h0 - first, 0); h < end; h += kBatch) {
            float u[kBatch][V], v[kBatch][V];
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                if (h + i < end) {
                    Vec<T>::load(x + (h + i) * a.D, u[i]);
                    Vec<T>::load(x + (h + i) * a.D + half, v[i]);
                }
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                if (h + i < end) {
                    float r[V], t[V];
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        r[e] = fmaf(u[i][e], cs[e], -(v[i][e] * sn[e]));
                        t[e] = fmaf(v[i][e], cs[e], u[i][e] * sn[e]);
                    }
                    Vec<T>::store(y + (h + i) * a.D, r);
                    Vec<T>::store(y + (h + i) * a.D + half, t);
                }
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
    k_rope_axes<T><<<dim3((unsigned)blocks, (unsigned)slices), dim3(x, tokens), 0, s>>>(a);
    note_launch();
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_rope_axes(const RopeAxesArgs &a, int dtype, cudaStream_t s)
{
    return dtype == RIS_F32 ? launch<float>(a, s) : launch<__nv_bfloat16>(a, s);
}

}  // namespace ris
