// The 4-bit cache: writing rows, reading them back, and one token's attention over them.
//
// A row (token, KV head) of D values is cut into groups of 32 with one bf16 scale
// bf16(max |x| * fl32(1/6)) each; a value is the e2m1 code (0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign) nearest to
// x / scale. Byte i of a row in natural order holds elements 2i (low half) and 2i + 1. Bytes are
// stored in the order in which the attention kernel's lanes take them, so that it unpacks a row
// without a shuffle (n = D / 32 groups, m = D / 16 tiles):
//   keys    word (4 bytes) u of group g goes to word u n + g: lane u of four takes its eighth-groups of all
//           groups with one load, elements 32 g + 8 u .. + 7;
//   values  byte c of 16-element tile e goes to byte c m + e: lane c of eight takes elements 16 e + 2 c and
//           + 1 of every tile with one load.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "attn_common.cuh"
#include "serve.h"

namespace ris {

// Device error word of this file (bit 1: tokens appended past the capacity).
__device__ unsigned int g_ris_cache4_error;

namespace {

// N elements in a row as they lie in memory, N * sizeof(T) a multiple of 4 and the address aligned to it
// (up to 16)
template <typename T, int N>
struct Raw {
    static constexpr int B = N * (int)sizeof(T), W = B >= 16 ? 16 : B;
    uint32_t w[B / 4];
    __device__ __forceinline__ void load(const T *p)
    {
#pragma unroll
        for (int i = 0; i < B / W; ++i) {
            const char *at = reinterpret_cast<const char *>(p) + i * W;
            if constexpr (W == 16) {
                const uint4 v = *reinterpret_cast<const uint4 *>(at);
                w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
            } else if constexpr (W == 8) {
                const uint2 v = *reinterpret_cast<const uint2 *>(at);
                w[2 * i] = v.x, w[2 * i + 1] = v.y;
            } else {
                w[i] = *reinterpret_cast<const uint32_t *>(at);
            }
        }
    }
    __device__ __forceinline__ float operator[](int e) const
    {
        if constexpr (sizeof(T) == 4)
            return __uint_as_float(w[e]);
        else
            return __uint_as_float((e & 1) ? (w[e >> 1] & 0xFFFF0000u) : (w[e >> 1] << 16));
    }
};

// |x| for a maximum that a NaN or an infinity must win: the bits without the sign
__device__ __forceinline__ uint32_t mag(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// The scale of a group whose largest magnitude has these bits; NaN where a value is not finite, so that
// the row then stands for NaN and no other row is touched
__device__ __forceinline__ __nv_bfloat16 scale_of(uint32_t top)
{
    return __float2bfloat16_rn(top >= 0x7F800000u ? __uint_as_float(0x7FFFFFFFu) : __uint_as_float(top) * (1.f / 6.f));
}

// the codes of a and b (a in the low half)
__device__ __forceinline__ uint32_t code2(float a, float b)
{
    uint16_t r;
    asm("{\n\t.reg .b8 t;\n\tcvt.rn.satfinite.e2m1x2.f32 t, %1, %2;\n\tcvt.u16.u8 %0, t;\n\t}" : "=h"(r) : "f"(b), "f"(a));
    return r;
}
// The codes of x / s, rounded to fp32 first as the format has it, without a division per value: with r =
// fl(1 / s), q = fl(x r) and the exact remainder x - q s, fl(q + r (x - q s)) is the quotient but for a
// relative 2^-46 before its one rounding (Markstein, IBM J. Res. Dev. 34, 1990). As the scale has 8
// significant bits, a quotient that is no fp32 number is at least 2^-33 of itself away from the middle of
// two, so the rounding is the division's own.
struct Scale {
    float s, r;
    bool plain;  // the scale is outside the range where no step over- or underflows
    __device__ __forceinline__ explicit Scale(float scale)
    {
        s = scale;
        r = 1.f / scale;
        plain = !(scale >= 0x1p-100f && scale <= 0x1p100f);
    }
    __device__ __forceinline__ float quotient(float x) const
    {
        const float q = x * r;
        return fmaf(fmaf(-q, s, x), r, q);
    }
    __device__ __forceinline__ uint32_t codes(float a, float b) const
    {
        if (plain) return s > 0.f ? code2(__fdiv_rn(a, s), __fdiv_rn(b, s)) : 0u;
        return code2(quotient(a), quotient(b));
    }
};

// Four lanes to a row of keys and its row of values; each lane loads what it stores (16 or 8 bytes of codes
// in one piece each), so rows are read and written in whole sectors; a group's maximum comes from its four
// lanes by shuffles. Bound by the latency of a row's chain (load, maximum, scale, codes: 350 instructions a
// lane) at the 32 warps that its registers leave an SM: 32,100 tokens of 2 heads of 128 take 11.5 us from
// L2, 15.5 from HBM, 8,028 CTAs over 8 heads 42 us at 4.0 TB/s. More warps with fewer registers (51, 42
// instead of 59) took 12.8 and 14.0 us, CTAs that stay and load ahead 14.4.
constexpr int kAppendThreads = 128;

template <typename T, int D>
__global__ void __launch_bounds__(kAppendThreads) k_cache4_append(const Cache4AppendArgs a)
{
    constexpr int NG = D / kCacheGroup, NM = D / 16;
    const int u = threadIdx.x & 3;
    const int64_t r = (int64_t)blockIdx.x * (kAppendThreads / 4) + threadIdx.x / 4;  // token and head
    const int64_t n_rows = a.total * a.c.Hkv;
    const bool in = r < n_rows;
    const int64_t r_in = in ? r : n_rows - 1;
    const int64_t tok = n_rows <= 0xFFFFFFFFLL ? (int64_t)((uint32_t)r_in / (uint32_t)a.c.Hkv) : r_in / a.c.Hkv;
    const int head = (int)(r_in - tok * a.c.Hkv);
    after_last();
    // lane u: the keys' elements 32 g + 8 u .. + 7 of every group, the values' 16 e + 4 u .. + 3 of every tile
    Raw<T, 8> xk[NG];
    Raw<T, 4> xv[NM];
    const T *pk = reinterpret_cast<const T *>(a.k) + tok * a.k_stride + head * D + 8 * u;
    const T *pv = reinterpret_cast<const T *>(a.v) + tok * a.v_stride + head * D + 4 * u;
#pragma unroll
    for (int g = 0; g < NG; ++g) xk[g].load(pk + kCacheGroup * g);
#pragma unroll
    for (int e = 0; e < NM; ++e) xv[e].load(pv + 16 * e);
    const int b = a.seq_of[tok], i = (int)tok - a.off[b];
    const int64_t slot = (int64_t)(a.start != nullptr ? a.start[b] : a.c.length[b]) + i;
    const bool ok = in && slot >= 0 && slot < a.c.cap;
    if (in && !ok) atomicOr(&g_ris_cache4_error, 2u);
    const int64_t row = ((int64_t)b * a.c.Hkv + head) * a.c.cap + slot;
    auto of_lanes = [](uint32_t top) {
        top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
        return max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
    };
    uint32_t wk[NG], wv[NM / 2], sk[NG], sv[NG];
#pragma unroll
    for (int g = 0; g < NG; ++g) {
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, mag(xk[g][e]));
        const __nv_bfloat16 s = scale_of(of_lanes(top));
        sk[g] = __bfloat16_as_ushort(s);
        const Scale sc(__bfloat162float(s));
        wk[g] = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) wk[g] |= sc.codes(xk[g][2 * e], xk[g][2 * e + 1]) << (8 * e);
    }
    // columns 2 u and 2 u + 1: NM bytes each, one per tile
#pragma unroll
    for (int w = 0; w < NM / 2; ++w) wv[w] = 0;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) top = max(top, max(mag(xv[2 * g][e]), mag(xv[2 * g + 1][e])));
        const __nv_bfloat16 s = scale_of(of_lanes(top));
        sv[g] = __bfloat16_as_ushort(s);
        const Scale sc(__bfloat162float(s));
#pragma unroll
        for (int e = 2 * g; e < 2 * g + 2; ++e)
#pragma unroll
            for (int c = 0; c < 2; ++c) wv[(c * NM + e) / 4] |= sc.codes(xv[e][2 * c], xv[e][2 * c + 1]) << (8 * (e & 3));
    }
    if (ok) {
        uint8_t *dk = a.c.k + row * (D / 2) + u * (4 * NG), *dv = a.c.v + row * (D / 2) + u * (2 * NM);
        if constexpr (D == 128) {
            *reinterpret_cast<uint4 *>(dk) = make_uint4(wk[0], wk[1], wk[2], wk[3]);
            *reinterpret_cast<uint4 *>(dv) = make_uint4(wv[0], wv[1], wv[2], wv[3]);
        } else {
            *reinterpret_cast<uint2 *>(dk) = make_uint2(wk[0], wk[1]);
            *reinterpret_cast<uint2 *>(dv) = make_uint2(wv[0], wv[1]);
        }
        if (u < 2) {
            uint32_t *ds = reinterpret_cast<uint32_t *>((u ? a.c.v_scale : a.c.k_scale) + row * NG);
#pragma unroll
            for (int g = 0; g < NG / 2; ++g) ds[g] = u ? sv[2 * g] | (sv[2 * g + 1] << 16) : sk[2 * g] | (sk[2 * g + 1] << 16);
        } else if (u == 2) {
            a.c.pos[row] = a.positions[tok];
        } else {
            a.c.weight[row] = a.weight != nullptr ? a.weight[(int64_t)head * a.total + tok] : 0.f;
        }
    }
    // the new lengths: written at once where the rows start at given slots, else by the last CTA,
    // once every CTA has read the old ones
    bool last = a.start != nullptr && blockIdx.x == 0;
    if (a.start == nullptr) {
        __shared__ bool done;
        __syncthreads();
        if (threadIdx.x == 0) {
            __threadfence();
            done = atomicAdd(a.ticket, 1u) == gridDim.x - 1;
            if (done) *a.ticket = 0u;
        }
        __syncthreads();
        last = done;
    }
    if (last)
        for (int s = threadIdx.x; s < a.c.B; s += kAppendThreads) {
            const int64_t n = (int64_t)(a.start != nullptr ? a.start[s] : a.c.length[s]) + (a.off[s + 1] - a.off[s]);
            a.c.length[s] = (int32_t)max((int64_t)0, min(n, a.c.cap));
        }
}

__global__ void __launch_bounds__(kAppendThreads) k_cache4_start(const Cache4Args c, const int32_t *start)
{
    const int s = blockIdx.x * kAppendThreads + threadIdx.x;
    after_last();
    if (s < c.B) c.length[s] = (int32_t)max((int64_t)0, min((int64_t)start[s], c.cap));
}

// the two values of a byte
__device__ __forceinline__ __half2 values2(uint32_t byte)
{
    uint32_t r;
    asm("{\n\t.reg .b8 t, z0, z1, z2;\n\tmov.b32 {t, z0, z1, z2}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, t;\n\t}" : "=r"(r) : "r"(byte));
    return *reinterpret_cast<const __half2 *>(&r);
}

// One thread per four elements of a row of the output, kReadRows rows of a list to a CTA: two bytes in, 16
// bytes out. Bound by the fp32 rows that it writes: 21 us for the 98 MB of two times 4 x 2 lists of 12,000
// slots of 128 (4.7 TB/s).
constexpr int kReadThreads = 256, kReadRows = 64;
template <int D>
__global__ void __launch_bounds__(kReadThreads) k_cache4_read(const Cache4Args c, const int32_t *first, int64_t count, int blocks,
                                                              float *ko, float *vo)
{
    constexpr int Q = D / 4, NG = D / kCacheGroup, NM = D / 16, STEP = kReadThreads / Q;
    const int64_t bh = blockIdx.x / blocks;
    after_last();
    const int64_t i0 = (int64_t)(blockIdx.x - bh * blocks) * kReadRows + threadIdx.x / Q;
    const int e = threadIdx.x % Q;  // elements 4 e .. 4 e + 3: bytes 2 e, 2 e + 1 in natural order
    const int b = (int)(bh / c.Hkv);
    const int64_t s0 = first != nullptr ? first[b] : 0, len = min((int64_t)c.length[b], c.cap);
    const bool values = blockIdx.y != 0;
    const int word = e / 2, tile = e / 4, col = 2 * (e & 3);
    const uint8_t *codes = (values ? c.v : c.k) + bh * c.cap * (D / 2) +
                           (values ? tile + col * NM : ((word & 3) * NG + (word >> 2)) * 4 + (e & 1) * 2);
    const uint16_t *scales = (values ? c.v_scale : c.k_scale) + bh * c.cap * NG + e / 8;
    float4 *out = reinterpret_cast<float4 *>(values ? vo : ko) + bh * count * Q + e;
#pragma unroll 4
    for (int64_t i = i0; i < min(count, i0 + kReadRows - (int)threadIdx.x / Q); i += STEP) {
        const int64_t slot = i + s0;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        if (slot >= 0 && slot < len) {
            const uint8_t *p = codes + slot * (D / 2);
            uint32_t b0, b1;
            if (values) {
                b0 = p[0], b1 = p[NM];
            } else {
                const uint32_t w = *reinterpret_cast<const uint16_t *>(p);
                b0 = w & 0xFFu, b1 = w >> 8;
            }
            const float sf = __uint_as_float((uint32_t)scales[slot * NG] << 16);
            const float2 lo = __half22float2(values2(b0)), hi = __half22float2(values2(b1));
            x = make_float4(lo.x * sf, lo.y * sf, hi.x * sf, hi.y * sf);
        }
        out[i * Q] = x;
    }
}

// ---------------------------------------------------------------- attention of one token
constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kTile = 16;                      // slots of a warp's product
constexpr int kUnit = kCacheUnit;              // slots by which the work is shared out
constexpr int kMostFactor = 127 + 118;         // largest factor of a weight times value scale (a weight is 2^8 at most), its exponent
constexpr int kMostHalf = 15;                  // what weight, scale and factor may come to as fp16 (log2)

template <int D, bool SPLIT>
struct Lay {
    static constexpr int TILES = SPLIT ? 2 : 4, SLOTS = TILES * kTile, STAGES = 8 / TILES;  // of a warp's stage; of its ring
    static constexpr int NG = D / kCacheGroup, NM = D / 16;
    static constexpr int CODES = D / 2, SCALES = 2 * NG;  // bytes of a slot
    static constexpr int OFF_K = 0, OFF_V = OFF_K + SLOTS * CODES, OFF_KS = OFF_V + SLOTS * CODES, OFF_VS = OFF_KS + SLOTS * SCALES,
                         STAGE = OFF_VS + SLOTS * SCALES;
    static constexpr int OFF_BARS = kWarps * STAGES * STAGE, BYTES = OFF_BARS + 8 * kWarps * STAGES;
    static_assert(kWarps * 8 * ((D + 4) * 4 + 12) <= OFF_BARS, "the warps' parts of a list pass through the rings");
};

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
constexpr int64_t kWaitLimit = int64_t(1) << 31;  // cycles
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, int64_t limit = kWaitLimit)
{
    const long long t0 = clock64();
    for (;;) {
        uint32_t ok;
        asm volatile(
            "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(bar), "r"(parity)
            : "memory");
        if (ok) return true;
        if (clock64() - t0 > limit) return false;
    }
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
                 "r"(bytes), "r"(bar)
                 : "memory");
}

__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// the product alone (no registers to clear for it)
__device__ __forceinline__ void mma0(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x)
{
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
// the values of a word's four bytes
__device__ __forceinline__ void unpack4(uint32_t w, uint32_t (&h)[4])
{
    asm("{\n\t.reg .b8 t0, t1, t2, t3;\n\tmov.b32 {t0, t1, t2, t3}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, t0;\n\tcvt.rn.f16x2.e2m1x2 %1, t1;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, t2;\n\tcvt.rn.f16x2.e2m1x2 %3, t3;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(w));
}
// the low (high) halves of every byte of a, and those of b as the high halves
__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return (a & 0x0F0F0F0Fu) | ((b << 4) & 0xF0F0F0F0u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return ((a >> 4) & 0x0F0F0F0Fu) | (b & 0xF0F0F0F0u); }
__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// two fp32 values in one register pair, and their product by halves
__device__ __forceinline__ uint64_t f2_pack(float x, float y)
{
    uint64_t d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(x), "f"(y));
    return d;
}
__device__ __forceinline__ void f2_unpack(uint64_t v, float &x, float &y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v)); }
__device__ __forceinline__ uint64_t f2_mul(uint64_t a, uint64_t b)
{
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint32_t pack_half(float x, float y)
{
    const __half2 h = __floats2half2_rn(x, y);
    return *reinterpret_cast<const uint32_t *>(&h);
}
// x - fp16(x), y - fp16(y) as fp16
__device__ __forceinline__ uint32_t pack_rest(float x, float y, uint32_t hi)
{
    const float2 h = __half22float2(*reinterpret_cast<const __half2 *>(&hi));
    return pack_half(x - h.x, y - h.y);
}
// 1 / f of a power of two, both normal numbers
__device__ __forceinline__ float inverse2(float f) { return __uint_as_float((254u << 23) - __float_as_uint(f)); }
__device__ __forceinline__ float bf16_at(uint32_t w, int e) { return __uint_as_float((e & 1) ? (w & 0xFFFF0000u) : (w << 16)); }

// Slot of row r (0 .. 15) of a tile: the rows that a lane needs as pairs along the product's inner
// dimension, 2 t, 2 t + 1, 2 t + 8 and 2 t + 9, are slots t, 4 + t, 8 + t and 12 + t, so that the four
// lanes t read neighbouring rows of the values.
__device__ __forceinline__ int tile_slot(int r) { return ((r & 7) >> 1) + 4 * (r & 1) + (r & 8); }

// How the slots in use are shared out. A list is a (sequence, KV head, block of 8 query heads) and holds
// ceil(length / kUnit) units; the units of all lists, one list after another, are cut into as many equal
// runs as there are CTAs, whatever the lengths are. CTA i's part of list l has partial number i + l: runs
// and lists advance together, so no two parts share a number. Lists of a sequence are neighbours: list = b
// * per_seq + y. Every warp works this out for itself, 32 sequences at a time by shuffles (with the block's
// barriers and 64-bit divisions it took 4 us).
__device__ __forceinline__ int64_t slots_of(const Cache4AttendArgs &a, int b)
{
    return max((int64_t)0, min((int64_t)a.c.length[b], a.reach));
}
__device__ __forceinline__ int64_t units_of(const Cache4AttendArgs &a, int b)
{
    return b < a.c.B ? (slots_of(a, b) + kUnit - 1) / kUnit : 0;
}
__device__ __forceinline__ int64_t warp_sum64(int64_t x)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
    return x;
}
// floor(x y / z)
__device__ __forceinline__ int64_t mul_div(int64_t x, int y, int z)
{
    return x < (1 << 20) && y < (1 << 11) ? (int64_t)((uint32_t)x * (uint32_t)y / (uint32_t)z) : x * y / z;
}

// Persistent CTAs of four warps; each CTA takes a run of units and the lists that it touches one after
// another. Its warps take stages of 64 slots (32 for fp32 outputs, whose accumulators double; fewer where
// that leaves warps without any) in turn, each with a softmax of its own over the slots that it saw and a
// ring of its own, filled by bulk copies (codes and scales are contiguous per KV head): no warp waits for
// another before a list's end. A tile of 16 slots:
//   S^T = K q^T  rows are slots, columns up to 8 query heads: the codes as fp16 (exact) straight from
//                the lane's word, one accumulator per group of 32, which the group's scale then multiplies in
//                fp32 (so the products are exact up to fp32 sums); the query as fp16 scaled by a power of
//                two, with a second fp16 of what that leaves for fp32 inputs;
//   O^T += V^T P^T  the weights times the slot's scale, per group of 32, as fp16, transposed by
//                movmatrix; with SPLIT a second fp16 of what the first leaves, for fp32 outputs; values as
//                fp16 pairs of slots, paired as codes (half the instructions of pairing them as fp16).
// The weights are p = 2^(s - m), m a whole number that moves only when a score exceeds it by more than 2^8;
// the row's sum is that of p alone, whatever the values hold. fp16 gets u = f p scale with a factor f, a
// power of two, per query head and group of 32 channels: it comes down when a u would pass 2^15, to where
// the largest of the stage is 16, and goes up with m, so what a slot adds keeps fp16's 11 bits down to
// 2^-18 of the largest that any slot so far has added to that head and group, and no group, slot or scale
// that is not finite takes bits from another group. O carries its group's f. Slots past the length enter
// with score -infinity and scale 0, whatever lies there. A list takes 8 query heads of its KV head, a
// product's columns: where a KV head has more, its slots are copied and unpacked once per 8.
// 16 sequences of 48,000 to 65,536 slots at 12 / 2 heads of 128, 258 MB: 52.0 us a call
// with the join, 5.0 of the 6.8 TB/s that a copy reaches (one exponent for all groups and heads, which a
// scale that is not finite or one large slot spoils, took 49.7; fp32 outputs 80 and 73); unpacking keeps
// the ALU pipe and the issue slots half busy, so three CTAs' loads and arithmetic do not overlap all the
// way. Smaller calls are latency: 24 sequences of 700 to 9,216 slots 16.3 us with the join (14.3
// with one exponent), of which the copies' first arrival and a warp's two stages are most.
constexpr float kLazyLog2 = 8.f;

template <typename T, bool SPLIT, int D>
__global__ void __launch_bounds__(kThreads, 3) k_cache4_attend(const Cache4AttendArgs a)
{
    using L = Lay<D, SPLIT>;
    constexpr int NG = L::NG, NM = L::NM, kWarpTiles = L::TILES, kStageSlots = L::SLOTS, kStages = L::STAGES;
    constexpr bool LO = sizeof(T) == 4;  // the query needs a second part
    extern __shared__ __align__(128) unsigned char smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g8 = lane >> 2, t4 = lane & 3;
    const int per_seq = a.lists / a.c.B;
    unsigned char *const ring = smem + warp * (kStages * L::STAGE);
    const uint32_t ring_at = smem_u32(ring), bars = smem_u32(smem) + L::OFF_BARS + 8 * kStages * warp;
    if (lane == 0) {
        for (int i = 0; i < kStages; ++i) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bars + 8 * i) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncwarp();
    after_last();  // (the join reads the lengths before it waits for this kernel)
    // this CTA's run of units, and the sequence that its first one is in
    int64_t total = 0;
    int64_t mine = units_of(a, lane);  // of the sequences that the search below looks at
    for (int b0 = 0; b0 < a.c.B; b0 += 32) total += warp_sum64(b0 == 0 ? mine : units_of(a, b0 + lane));
    total *= per_seq;
    const int ctas = (int)min((int64_t)gridDim.x, total);  // no run is empty
    if ((int)blockIdx.x >= ctas) return;
    int64_t at = mul_div(total, blockIdx.x, ctas);
    const int64_t end = mul_div(total, blockIdx.x + 1, ctas);
    int b = 0;
    int64_t base = 0;  // first unit of sequence b
    for (int b0 = 0;; b0 += 32) {
        if (b0 > 0) mine = units_of(a, b0 + lane);
        int64_t upto = mine * per_seq;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t x = __shfl_up_sync(0xFFFFFFFFu, upto, o);
            if (lane >= o) upto += x;
        }
        const uint32_t past = __ballot_sync(0xFFFFFFFFu, base + upto > at);
        if (past != 0u) {
            const int first = __ffs(past) - 1;
            b = b0 + first;
            base += __shfl_sync(0xFFFFFFFFu, upto - mine * per_seq, first);
            break;
        }
        base += __shfl_sync(0xFFFFFFFFu, upto, 31);  // (a sequence past `at` exists: at < total)
    }
    int used = 0, phase = 0;  // the warp's next stage of its ring, and the phase of its barrier
    bool ok = true;
    for (; b < a.c.B && at < end; ++b) {
        const int64_t len = slots_of(a, b), units = (len + kUnit - 1) / kUnit;
        if (units == 0) continue;
        // (below per_seq: at lies in this sequence)
        const int y0 = at - base <= 0xFFFFFFFFLL ? (int)((uint32_t)(at - base) / (uint32_t)units) : (int)((at - base) / units);
        base += y0 * units;
        for (int y = y0; y < per_seq && at < end; ++y, base += units) {
        const int64_t u1 = min(end, base + units);
        const int64_t first = (at - base) * kUnit;
        if (threadIdx.x == 0) {  // which CTAs' parts make up the list
            if (first == 0) a.list_cta[2 * ((int64_t)b * per_seq + y)] = (int)blockIdx.x;
            if (u1 == base + units) a.list_cta[2 * ((int64_t)b * per_seq + y) + 1] = (int)blockIdx.x;
        }
        const int n = (int)(min(len, (u1 - base) * kUnit) - first);  // slots of this part
        at = u1;
        const int kvh = y % a.c.Hkv, h0 = y / a.c.Hkv * 8;  // first head of the block
        const int nh = min(8, a.G - h0);
        const int64_t head0 = (int64_t)b * a.Hq + kvh * a.G + h0;
        const int64_t row0 = ((int64_t)b * a.c.Hkv + kvh) * a.c.cap + first;
        // the warp's stages: `per` slots from per (warp + 4 i) on
        const int per = min(kStageSlots, (n + kWarps * kTile - 1) / (kWarps * kTile) * kTile), s_step = kWarps * per;
        auto fetch = [&](int s0, int slot) {  // by one lane
            const int rows = min(per, (n - s0 + 15) / 16 * 16);
            const uint32_t bar = bars + 8 * slot, dst = ring_at + slot * L::STAGE;
            asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(rows * 2 * (L::CODES + L::SCALES))
                         : "memory");
            bulk_load(dst + L::OFF_K, a.c.k + (row0 + s0) * L::CODES, rows * L::CODES, bar);
            bulk_load(dst + L::OFF_KS, a.c.k_scale + (row0 + s0) * NG, rows * L::SCALES, bar);
            bulk_load(dst + L::OFF_V, a.c.v + (row0 + s0) * L::CODES, rows * L::CODES, bar);
            bulk_load(dst + L::OFF_VS, a.c.v_scale + (row0 + s0) * NG, rows * L::SCALES, bar);
        };
        // the queries: lane (g8, t4) holds elements 32 g + 8 t4 .. + 7 of head g8 of each block, scaled by 2^-e
        uint32_t qh[NG][4], ql[LO ? NG : 1][4];
        float unscale[2];  // of heads 2 t4, 2 t4 + 1: log2(e) / sqrt(D) 2^e
        {
            const int h = g8;
            const bool have = h < nh;
            const T *q = reinterpret_cast<const T *>(a.q) + (head0 + (have ? h : 0)) * D + 8 * t4;
            Raw<T, 8> x[NG];
#pragma unroll
            for (int g = 0; g < NG; ++g) x[g].load(q + kCacheGroup * g);
            // after the queries' loads: behind all the CTAs' copies, 30 MB at once, they would take 4 us
            // (the ring is empty here: the last part's stages were waited for, and its outputs have left it)
            if (lane == 0 && ok && !a.debug_no_loads)
                for (int i = 0, s0 = warp * per, slot = used; i < kStages && s0 < n; ++i, s0 += s_step) {
                    fetch(s0, slot);
                    slot = slot + 1 == kStages ? 0 : slot + 1;
                }
            uint32_t top = 0;
#pragma unroll
            for (int g = 0; g < NG; ++g)
#pragma unroll
                for (int e = 0; e < 8; ++e) top = max(top, mag(x[g][e]));
            top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
            top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
            // |q| 2^-e below 2^13; the exponent stays where both factors are normal numbers
            const int e2 = min(max((int)(top >> 23) - 127 - 12, -100), 100);
            const float down = pow2i(-e2), up = pow2i(e2) * a.scale_log2;
#pragma unroll
            for (int g = 0; g < NG; ++g)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float u = have ? x[g][2 * e] * down : 0.f, v = have ? x[g][2 * e + 1] * down : 0.f;
                    qh[g][e] = pack_half(u, v);
                    if constexpr (LO) ql[g][e] = pack_rest(u, v, qh[g][e]);
                }
            unscale[0] = __shfl_sync(0xFFFFFFFFu, up, 8 * t4);
            unscale[1] = __shfl_sync(0xFFFFFFFFu, up, 8 * t4 + 4);
        }
        float m[2], l[2], fac[2][NG], o[NM][4];  // (index 0, 1: heads 2 t4, 2 t4 + 1)
        {
            m[0] = m[1] = -INFINITY;
            l[0] = l[1] = 0.f;
#pragma unroll
            for (int g = 0; g < NG; ++g) fac[0][g] = fac[1][g] = __uint_as_float((uint32_t)kMostFactor << 23);
#pragma unroll
            for (int e = 0; e < NM; ++e) o[e][0] = o[e][1] = o[e][2] = o[e][3] = 0.f;
        }
        // a stage of ns slots at s0; FULL: ns == kStageSlots
        auto stage = [&](auto full_c, const unsigned char *sm, int s0, int ns) {
            constexpr bool FULL = decltype(full_c)::value;
            // the value scales of this lane's slots, two groups to a word, and the largest
            uint32_t vsc[kWarpTiles][2][NG / 2], top[NG / 2] = {};
#pragma unroll
            for (int i = 0; i < kWarpTiles; ++i)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const int slot = i * kTile + tile_slot(g8 + 8 * r);
                    const uint32_t *p = reinterpret_cast<const uint32_t *>(sm + L::OFF_VS + slot * L::SCALES);
#pragma unroll
                    for (int g = 0; g < NG / 2; ++g) {
                        vsc[i][r][g] = FULL || slot < ns ? p[g] : 0u;
                        top[g] = __vmaxu2(top[g], vsc[i][r][g]);
                    }
                }
            {
                float s[kWarpTiles][4];
#pragma unroll
                for (int i = 0; i < kWarpTiles; ++i) {
                    if (!FULL && i * kTile >= ns) {
                        s[i][0] = s[i][1] = s[i][2] = s[i][3] = -INFINITY;
                        continue;
                    }
                    uint32_t kw[2][NG], ksw[2][NG / 2];
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const int slot = i * kTile + tile_slot(g8 + 8 * r);
                        const unsigned char *p = sm + L::OFF_K + slot * L::CODES + t4 * (4 * NG);
                        const uint32_t *ps = reinterpret_cast<const uint32_t *>(sm + L::OFF_KS + slot * L::SCALES);
                        if constexpr (NG == 4) {
                            const uint4 w = *reinterpret_cast<const uint4 *>(p);
                            kw[r][0] = w.x, kw[r][1] = w.y, kw[r][2] = w.z, kw[r][3] = w.w;
                        } else {
                            const uint2 w = *reinterpret_cast<const uint2 *>(p);
                            kw[r][0] = w.x, kw[r][1] = w.y;
                        }
#pragma unroll
                        for (int g = 0; g < NG / 2; ++g) ksw[r][g] = ps[g];
                    }
                    float acc[4] = {};
#pragma unroll
                    for (int g = 0; g < NG; ++g) {
                        uint32_t x[4], z[4];
                        unpack4(kw[0][g], x);
                        unpack4(kw[1][g], z);
                        float d[4];
                        const uint32_t f0[4] = {x[0], z[0], x[1], z[1]}, f1[4] = {x[2], z[2], x[3], z[3]};
                        mma0(d, f0, qh[g][0], qh[g][1]);
                        mma(d, f1, qh[g][2], qh[g][3]);
                        if constexpr (LO) {
                            mma(d, f0, ql[g][0], ql[g][1]);
                            mma(d, f1, ql[g][2], ql[g][3]);
                        }
                        const float k0 = bf16_at(ksw[0][g / 2], g), k1 = bf16_at(ksw[1][g / 2], g);
                        acc[0] = g == 0 ? d[0] * k0 : fmaf(d[0], k0, acc[0]);
                        acc[1] = g == 0 ? d[1] * k0 : fmaf(d[1], k0, acc[1]);
                        acc[2] = g == 0 ? d[2] * k1 : fmaf(d[2], k1, acc[2]);
                        acc[3] = g == 0 ? d[3] * k1 : fmaf(d[3], k1, acc[3]);
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        s[i][e] = acc[e];
                        if (!FULL && i * kTile + tile_slot(g8 + 8 * (e >> 1)) >= ns) s[i][e] = -INFINITY;
                    }
                    if (a.scores != nullptr) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int h = 2 * t4 + (e & 1), slot = i * kTile + tile_slot(g8 + 8 * (e >> 1));
                            if ((FULL || slot < ns) && h < nh)
                                a.scores[(head0 + h) * a.score_pitch + first + s0 + slot] = s[i][e] * unscale[e & 1];
                        }
                    }
                }
                float x[2];
                bool moves = false;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    x[e] = fmaxf(s[0][e], s[0][e + 2]);
#pragma unroll
                    for (int i = 1; i < kWarpTiles; ++i) x[e] = fmaxf(x[e], fmaxf(s[i][e], s[i][e + 2]));
                    x[e] *= unscale[e];
                    // no u of this lane is larger than its largest weight times its largest scales, all
                    // groups' together (NaN: not known to be small)
                    float most = 0.f;
#pragma unroll
                    for (int g = 0; g < NG; ++g) most = fmaf(fac[e][g], bf16_at(top[g / 2], g), most);
                    moves = moves || x[e] > m[e] + kLazyLog2 || !(ex2(x[e] - m[e]) * most <= (float)(1 << kMostHalf));
                }
                if (__any_sync(0xFFFFFFFFu, moves)) {  // (in the first stages of a list, mostly)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
#pragma unroll
                        for (int w = 4; w < 32; w <<= 1) x[e] = fmaxf(x[e], __shfl_xor_sync(0xFFFFFFFFu, x[e], w));
                        const bool begun = m[e] != -INFINITY;  // (else O and l are 0, or NaN)
                        int up = 0;
                        if (x[e] > m[e] + kLazyLog2) {
                            const float nm = ceilf(x[e]);
                            if (begun) {
                                l[e] *= ex2(m[e] - nm);
                                up = (int)fminf(nm - m[e], 1000.f);
                            }
                            m[e] = nm;
                        }
                        const float ref = m[e] == -INFINITY ? 0.f : m[e];
                        // largest weight times scale, times 2^-8, of two groups in a word: its power of two is what counts, which
                        // bf16 gives (a NaN is passed over)
                        __nv_bfloat162 most[NG / 2];
#pragma unroll
                        for (int g = 0; g < NG / 2; ++g) most[g] = __float2bfloat162_rn(0.f);
#pragma unroll
                        for (int i = 0; i < kWarpTiles; ++i)
#pragma unroll
                            for (int r = 0; r < 2; ++r) {
                                const __nv_bfloat162 p = __float2bfloat162_rn(ex2(fmaf(s[i][e + 2 * r], unscale[e], -ref)) * 0x1p-8f);
#pragma unroll
                                for (int g = 0; g < NG / 2; ++g)
                                    most[g] = __hmax2(most[g], __hmul2(p, *reinterpret_cast<const __nv_bfloat162 *>(&vsc[i][r][g])));
                            }
#pragma unroll
                        for (int g = 0; g < NG / 2; ++g)
#pragma unroll
                            for (int w = 4; w < 32; w <<= 1) most[g] = __hmax2(most[g], __shfl_xor_sync(0xFFFFFFFFu, most[g], w));
#pragma unroll
                        for (int g = 0; g < NG; ++g) {
                            // by exponents (of 127 + the power): the factor goes up as the weights come down, where O stays as it
                            // is, and comes down to where the largest product is 16
                            const int top = (int)(__float_as_uint(bf16_at(*reinterpret_cast<const uint32_t *>(&most[g / 2]), g)) >> 23);
                            const int had = (int)(__float_as_uint(fac[e][g]) >> 23) + up;
                            int now = min(had, kMostFactor);
                            if (top + now - 2 * 127 >= kMostHalf - 8) now = max(1, 2 * 127 - 4 - top);
                            fac[e][g] = __uint_as_float((uint32_t)now << 23);
                            if (begun && now != had) {
                                const float by = now - had < -126 ? 0.f : pow2i(now - had);
#pragma unroll
                                for (int t = 2 * g; t < 2 * g + 2; ++t) {
                                    o[t][e] *= by;
                                    o[t][e + 2] *= by;
                                }
                            }
                        }
                    }
                }
                // fp32 outputs: the stage's products from zero, added to O in fp32 afterwards. (The tensor
                // pipe's additions cut off: over thousands of slots in one accumulator 2e-6 of the result.)
                [[maybe_unused]] float part[SPLIT ? NM : 1][4];
                const float to[2] = {m[0] == -INFINITY ? 0.f : -m[0], m[1] == -INFINITY ? 0.f : -m[1]};  // exponent of a weight: s unscale + to
#pragma unroll
                for (int i = 0; i < kWarpTiles; ++i) {
                    if (!FULL && i * kTile >= ns) continue;
                    float p[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        p[e] = ex2(fmaf(s[i][e], unscale[e & 1], to[e & 1]));
                        l[e & 1] += p[e];
                    }
                    [[maybe_unused]] uint32_t bh[NG][2], bl[SPLIT ? NG : 1][2];
#pragma unroll
                    for (int r = 0; r < 2; ++r)
#pragma unroll
                        for (int g = 0; g < NG; ++g) {
                            const float sc = bf16_at(vsc[i][r][g / 2], g);
                            float u, v;
                            f2_unpack(f2_mul(f2_mul(f2_pack(p[2 * r], p[2 * r + 1]), f2_pack(fac[0][g], fac[1][g])), f2_pack(sc, sc)), u, v);
                            const uint32_t hi = pack_half(u, v);
                            if constexpr (SPLIT) bl[g][r] = transpose8(pack_rest(u, v, hi));
                            bh[g][r] = transpose8(hi);
                        }
                    uint32_t vw[4][NM / 4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const unsigned char *p8 = sm + L::OFF_V + (i * kTile + 4 * r + t4) * L::CODES + g8 * NM;
                        if constexpr (NM == 8) {
                            const uint2 w = *reinterpret_cast<const uint2 *>(p8);
                            vw[r][0] = w.x, vw[r][1] = w.y;
                        } else {
                            vw[r][0] = *reinterpret_cast<const uint32_t *>(p8);
                        }
                    }
#pragma unroll
                    for (int q4 = 0; q4 < NM / 4; ++q4) {
                        // byte e of the words x (slots of rows 2 t, 2 t + 1) and y (2 t + 8, 2 t + 9): the
                        // pair of values of element 2 g8 (index 0) or 2 g8 + 1 (1) of tile 4 q4 + e
                        uint32_t x[2][4], y[2][4];
                        unpack4(low_halves(vw[0][q4], vw[1][q4]), x[0]);
                        unpack4(high_halves(vw[0][q4], vw[1][q4]), x[1]);
                        unpack4(low_halves(vw[2][q4], vw[3][q4]), y[0]);
                        unpack4(high_halves(vw[2][q4], vw[3][q4]), y[1]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int tl = 4 * q4 + e;
                            const uint32_t f[4] = {x[0][e], x[1][e], y[0][e], y[1][e]};
                            if constexpr (SPLIT) {
                                if (i == 0)
                                    mma0(part[tl], f, bl[tl / 2][0], bl[tl / 2][1]);
                                else
                                    mma(part[tl], f, bl[tl / 2][0], bl[tl / 2][1]);
                                mma(part[tl], f, bh[tl / 2][0], bh[tl / 2][1]);
                            } else {
                                mma(o[tl], f, bh[tl / 2][0], bh[tl / 2][1]);
                            }
                        }
                    }
                }
                if constexpr (SPLIT) {
#pragma unroll
                    for (int e = 0; e < NM; ++e)
#pragma unroll
                        for (int c = 0; c < 4; ++c) o[e][c] += part[e][c];
                }
            }
        };
        for (int s0 = warp * per; ok && s0 < n; s0 += s_step) {
            ok = __all_sync(0xFFFFFFFFu, mbar_wait(bars + 8 * used, phase, a.wait_limit));
            if (!ok) {
                // the stages asked for, this one and the next of the ring, have landed before the ring is
                // used for anything else, or the CTA ends
                for (int i = 0; i < kStages && s0 < n && !a.debug_no_loads; ++i, s0 += s_step) {
                    mbar_wait(bars + 8 * used, phase);
                    if (++used == kStages) used = 0, phase ^= 1;
                }
                break;
            }
            const unsigned char *sm = ring + used * L::STAGE;
            if (min(per, n - s0) == kStageSlots)
                stage(std::true_type{}, sm, s0, kStageSlots);
            else
                stage(std::false_type{}, sm, s0, min(per, n - s0));
            __syncwarp();  // every lane is done with the stage
            if (lane == 0 && s0 + kStages * s_step < n) fetch(s0 + kStages * s_step, used);
            if (++used == kStages) used = 0, phase ^= 1;
        }
        __syncwarp();
        // the four warps' parts of each head, through the rings: [warp][head][D], (maximum, sum), factors
        __syncthreads();
        constexpr int LO_ = D + 4;  // (the four lanes t4 write rows two apart)
        float *const so = reinterpret_cast<float *>(smem);
        float2 *const sml = reinterpret_cast<float2 *>(so + kWarps * 8 * LO_);
        float *const sf = reinterpret_cast<float *>(sml + kWarps * 8);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float x = l[e];
#pragma unroll
            for (int w = 4; w < 32; w <<= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, w);
            const int h = 2 * t4 + e;
            const float inv = x == 0.f ? 0.f : 1.f / x;  // (averages: sums of the largest values would pass fp32's range)
            if (g8 == 0) sml[warp * 8 + h] = make_float2(m[e], x);
#pragma unroll
            for (int tl = 0; tl < NM; ++tl)
                *reinterpret_cast<float2 *>(so + (warp * 8 + h) * LO_ + 16 * tl + 2 * g8) =
                    make_float2(o[tl][e] * inv * inverse2(fac[e][tl / 2]), o[tl][e + 2] * inv * inverse2(fac[e][tl / 2]));
        }
        __syncthreads();
        // one partial per head of the block: number cta + list
        const int64_t part = ((int64_t)blockIdx.x + (int64_t)b * per_seq + y) * 8;
        if (warp == 0) {  // lane: warp lane / 8, head lane mod 8
            const float2 ml = sml[lane];
            float M = fmaxf(ml.x, __shfl_xor_sync(0xFFFFFFFFu, ml.x, 8));
            M = fmaxf(M, __shfl_xor_sync(0xFFFFFFFFu, M, 16));
            const float part_sum = ml.y * (ml.x == -INFINITY ? 0.f : exp2f(ml.x - M));
            float sum = part_sum + __shfl_xor_sync(0xFFFFFFFFu, part_sum, 8);
            sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 16);
            sf[lane] = sum == 0.f ? 0.f : part_sum / sum;  // the warp's share of the average
            if (lane < nh) a.part_ml[part + lane] = make_float2(M, sum);
        }
        __syncthreads();
        for (int t = threadIdx.x; t < nh * (D / 4); t += kThreads) {
            const int h = t / (D / 4), d = t % (D / 4) * 4;
            float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float f = sf[w * 8 + h];
                const float4 v = *reinterpret_cast<const float4 *>(so + (w * 8 + h) * LO_ + d);
                x.x = fmaf(v.x, f, x.x), x.y = fmaf(v.y, f, x.y), x.z = fmaf(v.z, f, x.z), x.w = fmaf(v.w, f, x.w);
            }
            *reinterpret_cast<float4 *>(a.part_o + (part + h) * D + d) = x;
        }
        // the rings take copies again: after every read of them, and ordered before them
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncthreads();
        }
    }
    if (!ok) atomicOr(&g_ris_cache4_error, 4u);  // (a copy that was given up: the outputs are undefined)
}

// Joins the parts of a list. The first CTAs: one per (query head, sequence), warps over its parts, a lane
// per channels; then (weights) CTAs that add up what each slot got from the heads of its KV head, from the
// scores that the first kernel left. Launched as its programmatic dependent. Latency: 8 us with the weights
// of 24 x 2 lists of 700 to 9,216 slots, 7 MB of scores.
constexpr int kJoinWarps = 4, kJoinThreads = 32 * kJoinWarps;
constexpr int kWeightSlots = 4 * kJoinThreads;  // slots of a CTA

template <typename TO, int D>
__global__ void __launch_bounds__(kJoinThreads) k_cache4_join(const Cache4AttendArgs a)
{
    constexpr int C = D / 32, block_heads = 8;
    __shared__ float so[kJoinWarps][D];
    __shared__ float2 sml[kJoinWarps];
    extern __shared__ float2 stat[];  // [G], weights
    const int b = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int per_seq = a.lists / a.c.B;
    const int64_t len = slots_of(a, b);
    // a CTA of the weights: its KV head and this thread's four slots
    const int w = (int)blockIdx.x - a.Hq, blocks = ((int)gridDim.x - a.Hq) / a.c.Hkv, kvh_w = w >= 0 ? w / blocks : 0;
    const int64_t s0 = (int64_t)(w >= 0 ? w % blocks : 0) * kWeightSlots;
    if (w >= 0 && s0 >= len) return;  // (the CTAs of the outputs wait for the first kernel in any case)
    after_last();
    // the parts of list y of this sequence: CTAs i0 .. i1, partial numbers i + list
    auto parts = [&](int y, int &i0, int &i1) {
        const int2 x = reinterpret_cast<const int2 *>(a.list_cta)[(int64_t)b * per_seq + y];
        i0 = len > 0 ? x.x : 0;
        i1 = len > 0 ? x.y : -1;
    };
    if ((int)blockIdx.x < a.Hq) {
        const int h = blockIdx.x, kvh = h / a.G, hb = (h % a.G) / block_heads, y = hb * a.c.Hkv + kvh;
        int i0, i1;
        parts(y, i0, i1);
        const int64_t p0 = ((int64_t)b * per_seq + y) * block_heads + h % a.G % block_heads;
        // (averages, so that sums of values do not pass fp32's range, times sums of weights that may be as many as there
        // are slots: scaled down)
        constexpr float kDown = 0x1p-20f;
        float M = -INFINITY, sum = 0.f, x[C] = {};
#pragma unroll 4
        for (int i = i0 + warp; i <= i1; i += kJoinWarps) {
            const int64_t p = p0 + (int64_t)i * block_heads;
            const float2 ml = a.part_ml[p];
            float v[C];
#pragma unroll
            for (int c = 0; c < C; ++c) v[c] = a.part_o[p * D + lane + 32 * c];
            const float nm = fmaxf(M, ml.x);
            const float f0 = M == -INFINITY ? 0.f : exp2f(M - nm), f1 = ml.y * (ml.x == -INFINITY ? 0.f : exp2f(ml.x - nm));
            M = nm;
            sum = fmaf(sum, f0, f1);
#pragma unroll
            for (int c = 0; c < C; ++c) x[c] = fmaf(x[c], f0, v[c] * (f1 * kDown));
        }
        if (lane == 0) sml[warp] = make_float2(M, sum);
#pragma unroll
        for (int c = 0; c < C; ++c) so[warp][lane + 32 * c] = x[c];
        __syncthreads();
        const int64_t row = (int64_t)b * a.Hq + h;
        const int d = threadIdx.x;
        if (d < D) {
            float tm = -INFINITY, ts = 0.f, to = 0.f;
#pragma unroll
            for (int w = 0; w < kJoinWarps; ++w) tm = fmaxf(tm, sml[w].x);
#pragma unroll
            for (int w = 0; w < kJoinWarps; ++w) {
                const float f = sml[w].x == -INFINITY ? 0.f : exp2f(sml[w].x - tm);
                ts = fmaf(sml[w].y, f, ts);
                to = fmaf(so[w][d], f, to);
            }
            to = ts == 0.f ? 0.f : to / (ts * kDown);  // no slot: zeros
            if constexpr (sizeof(TO) == 4)
                reinterpret_cast<float *>(a.out)[row * D + d] = to;
            else
                reinterpret_cast<__nv_bfloat16 *>(a.out)[row * D + d] = __float2bfloat16_rn(to);
            if (d == 0 && a.lse != nullptr) a.lse[row] = (tm + log2f(ts)) * kLn2;
        }
        return;
    }
    // weights: the scores of the first eight heads are on their way before the heads' sums are known
    const int64_t s1 = s0 + 4 * threadIdx.x, row = ((int64_t)b * a.c.Hkv + kvh_w) * a.c.cap + s1;
    const float *sc = a.scores + ((int64_t)b * a.Hq + kvh_w * a.G) * a.score_pitch + s1;
    const bool in = s1 < len;
    float4 x[8], y = make_float4(0.f, 0.f, 0.f, 0.f);
    auto load = [&](int h0) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (in && h0 + e < a.G) x[e] = *reinterpret_cast<const float4 *>(sc + (h0 + e) * a.score_pitch);
    };
    load(0);
    if (in && a.weight_in != nullptr) y = *reinterpret_cast<const float4 *>(a.weight_in + row);
    for (int h = warp; h < a.G; h += kJoinWarps) {  // a warp per head, a lane per part
        const int yl = h / block_heads * a.c.Hkv + kvh_w;
        int i0, i1;
        parts(yl, i0, i1);
        const int64_t p0 = ((int64_t)b * per_seq + yl) * block_heads + h % block_heads;
        float M = -INFINITY, sum = 0.f;
        for (int i = i0 + lane; i <= i1; i += 32) {
            const float2 ml = a.part_ml[p0 + (int64_t)i * block_heads];
            const float nm = fmaxf(M, ml.x);
            sum = nm == -INFINITY ? sum + ml.y : sum * exp2f(M - nm) + ml.y * exp2f(ml.x - nm);
            M = nm;
        }
        const float tm = warp_max(M);
        sum = warp_sum(tm == -INFINITY ? sum : sum * exp2f(M - tm));
        if (lane == 0) stat[h] = make_float2(tm, 1.f / sum);
    }
    __syncthreads();
    for (int h0 = 0; h0 < a.G; h0 += 8) {
        if (h0 > 0) load(h0);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (in && h0 + e < a.G) {
                const float2 ml = stat[h0 + e];
                y.x = fmaf(ex2(x[e].x - ml.x), ml.y, y.x);
                y.y = fmaf(ex2(x[e].y - ml.x), ml.y, y.y);
                y.z = fmaf(ex2(x[e].z - ml.x), ml.y, y.z);
                y.w = fmaf(ex2(x[e].w - ml.x), ml.y, y.w);
            }
    }
    if (s1 + 4 <= len) {
        *reinterpret_cast<float4 *>(a.weight_out + row) = y;
    } else if (in) {  // slots past the length stay as they are
        const float z[4] = {y.x, y.y, y.z, y.w};
        for (int e = 0; e < (int)(len - s1); ++e) a.weight_out[row + e] = z[e];
    }
}

template <typename T, bool SPLIT, int D>
cudaError_t launch_part(const Cache4AttendArgs &a, cudaStream_t s)
{
    auto kern = k_cache4_attend<T, SPLIT, D>;
    constexpr int bytes = Lay<D, SPLIT>::BYTES;
    static Once once;
    const cudaError_t ready = once([&] { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes); });
    if (ready != cudaSuccess) return ready;
    return launch_chained(kern, dim3((unsigned)a.ctas), dim3(kThreads), bytes, s, a);
}
template <typename T, bool SPLIT>
cudaError_t launch_part_d(const Cache4AttendArgs &a, cudaStream_t s)
{
    return a.c.D == 128 ? launch_part<T, SPLIT, 128>(a, s) : launch_part<T, SPLIT, 64>(a, s);
}
template <typename TO, int D>
cudaError_t launch_join_d(const Cache4AttendArgs &a, cudaStream_t s)
{
    const int64_t blocks = a.weight_out != nullptr ? (a.reach + kWeightSlots - 1) / kWeightSlots * a.c.Hkv : 0;
    return launch_chained(k_cache4_join<TO, D>, dim3((unsigned)(a.Hq + blocks), (unsigned)a.c.B), dim3(kJoinThreads),
                          a.weight_out != nullptr ? a.G * sizeof(float2) : 0, s, a);
}
template <typename TO>
cudaError_t launch_join(const Cache4AttendArgs &a, cudaStream_t s)
{
    return a.c.D == 128 ? launch_join_d<TO, 128>(a, s) : launch_join_d<TO, 64>(a, s);
}

}  // namespace

cudaError_t launch_cache4_append(const Cache4AppendArgs &a, int dtype, cudaStream_t s)
{
    const int64_t rows = a.total * a.c.Hkv, per = kAppendThreads / 4;
    const dim3 grid((unsigned)((rows + per - 1) / per)), block(kAppendThreads);
    if (dtype == RIS_F32)
        return a.c.D == 128 ? launch_chained(k_cache4_append<float, 128>, grid, block, 0, s, a)
                            : launch_chained(k_cache4_append<float, 64>, grid, block, 0, s, a);
    return a.c.D == 128 ? launch_chained(k_cache4_append<__nv_bfloat16, 128>, grid, block, 0, s, a)
                        : launch_chained(k_cache4_append<__nv_bfloat16, 64>, grid, block, 0, s, a);
}

cudaError_t launch_cache4_start(const Cache4Args &c, const int32_t *start, cudaStream_t s)
{
    return launch_chained(k_cache4_start, dim3((unsigned)((c.B + kAppendThreads - 1) / kAppendThreads)), dim3(kAppendThreads), 0, s, c, start);
}

cudaError_t launch_cache4_read(const Cache4Args &c, const int32_t *first, int64_t count, float *k, float *v, cudaStream_t s)
{
    const int blocks = (int)((count + kReadRows - 1) / kReadRows);
    const dim3 grid((unsigned)((int64_t)c.B * c.Hkv * blocks), 2), block(kReadThreads);
    return c.D == 128 ? launch_chained(k_cache4_read<128>, grid, block, 0, s, c, first, count, blocks, k, v)
                      : launch_chained(k_cache4_read<64>, grid, block, 0, s, c, first, count, blocks, k, v);
}

cudaError_t launch_cache4_attend(Cache4AttendArgs a, int dtype, int out_dtype, cudaStream_t s)
{
    if (a.wait_limit == 0) a.wait_limit = kWaitLimit;
    // fp32 outputs take the weights as two fp16 parts (22 bits), bf16 outputs as one (11 bits, against the
    // 8 that the output keeps)
    cudaError_t e;
    if (dtype == RIS_F32)
        e = out_dtype == RIS_F32 ? launch_part_d<float, true>(a, s) : launch_part_d<float, false>(a, s);
    else
        e = out_dtype == RIS_F32 ? launch_part_d<__nv_bfloat16, true>(a, s) : launch_part_d<__nv_bfloat16, false>(a, s);
    if (e != cudaSuccess) return e;
    return out_dtype == RIS_F32 ? launch_join<float>(a, s) : launch_join<__nv_bfloat16>(a, s);
}

cudaError_t cache4_error_word(unsigned int **p) { return cudaGetSymbolAddress(reinterpret_cast<void **>(p), g_ris_cache4_error); }

}  // namespace ris
