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

// The same by half turns: the fraction's top 24 bits exactly, the next 32 as a turn by so small an angle (2^-23 half turns at most) that
// its cosine is 1. The 24 bits alone would be off by up to 9e-8 radians, as an angle rounded to fp32 is.
__device__ __forceinline__ void sincos_half_turns(int32_t p, uint64_t turn, float *sn, float *cs)
{
    const int64_t frac = (int64_t)(turn * (uint64_t)(int64_t)p);
    float s, c;
    sincospif((float)(int32_t)(frac >> 40) * 0x1p-23f, &s, &c);
    const float rest = (float)(uint32_t)(frac >> 8) * (3.14159265f * 0x1p-55f);
    *sn = fmaf(c, rest, s);
    *cs = fmaf(s, -rest, c);
}

}  // namespace rows
}  // namespace ris
