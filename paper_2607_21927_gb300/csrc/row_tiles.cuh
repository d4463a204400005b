// A tile of 128 query rows against 128 keys in tensor memory, one row to a thread: what the attention
// kernels that work that way share.
#pragma once

#include <cudaTypedefs.h>
#include <cuda_runtime.h>

#include <mutex>

#include "tcgen05.cuh"

namespace ris {
namespace tc {

constexpr int kTileRows = 128, kTileKeys = 128;

// The driver's encoder of tensor maps, or null.
inline PFN_cuTensorMapEncodeTiled_v12000 encode_fn()
{
    static std::once_flag once;
    static PFN_cuTensorMapEncodeTiled_v12000 fn = nullptr;
    std::call_once(once, [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
    });
    return fn;
}

// kept keys of word e of a tile, as bits: those up to the row's last one (counted from the tile's start)
__device__ __forceinline__ uint32_t causal_word(int last, int e)
{
    const int lim = min(31, max(-1, last - 32 * e));
    return lim < 0 ? 0u : 0xFFFFFFFFu >> (31 - lim);
}
// x = -infinity unless the word has the bit: a predicated move
__device__ __forceinline__ void drop_unless(float &x, uint32_t word, uint32_t bit)
{
    asm("{\n\t.reg .pred p;\n\t.reg .b32 t;\n\t"
        "and.b32 t, %1, %2;\n\tsetp.eq.u32 p, t, 0;\n\t@p mov.b32 %0, 0xFF800000;\n\t}"
        : "+f"(x)
        : "r"(word), "r"(bit));
}
template <int BN>
__device__ __forceinline__ float row_max(const float (&sv)[BN])
{
    float mx8[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        mx8[e] = fmaxf(sv[e], sv[e + 8]);
#pragma unroll
        for (int c = 16; c < BN; c += 16) mx8[e] = fmax3(mx8[e], sv[c + e], sv[c + 8 + e]);
    }
    return fmax3(fmax3(mx8[0], mx8[1], mx8[2]), fmax3(mx8[3], mx8[4], mx8[5]), fmaxf(mx8[6], mx8[7]));
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}
// 16 bytes of outputs (four fp32 or eight bf16 values)
template <typename TOut>
__device__ __forceinline__ void store16(void *dst, const float *x)
{
    if constexpr (sizeof(TOut) == 4)
        *reinterpret_cast<float4 *>(dst) = make_float4(x[0], x[1], x[2], x[3]);
    else
        *reinterpret_cast<uint4 *>(dst) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}

}  // namespace tc
}  // namespace ris
