// What the kernels that turn heads to their positions share.
#pragma once

#include <cuda_bf16.h>

#include <cstdint>

namespace ris {
namespace rows {

// 16 bytes of elements
template <typename T>
struct Vec {
    static constexpr int V = 16 / (int)sizeof(T);
    uint4 raw;
    __device__ __forceinline__ void load(const T *p) { raw = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ float operator[](int e) const
    {
        const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
        if constexpr (V == 4)
            return __uint_as_float(w[e]);
        else
            return __uint_as_float((e & 1) ? (w[e >> 1] & 0xFFFF0000u) : (w[e >> 1] << 16));
    }
    static __device__ __forceinline__ void store(T *p, const float *x)
    {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (V == 4) {
                w[e] = __float_as_uint(x[e]);
            } else {
                const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * e], x[2 * e + 1]);
                w[e] = *reinterpret_cast<const uint32_t *>(&b);
            }
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

// The same with the fraction's top 32 bits as half turns, rounded to 24 bits (pi 2^-25 radians at most, like the rounding of
// an angle in fp32): fewer instructions, 3.0 instead of 3.5 us where a call is one chain of latencies.
__device__ __forceinline__ void sincos_half_turns(int32_t p, uint64_t turn, float *sn, float *cs)
{
    const int32_t top = (int32_t)(turn * (uint64_t)(int64_t)p >> 32);
    sincospif((float)top * 0x1p-31f, sn, cs);
}

}  // namespace rows
}  // namespace ris
