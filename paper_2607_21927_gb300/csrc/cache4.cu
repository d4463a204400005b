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

#include "attn_common.cuh"
#include "serve.h"

namespace ris {

// Device error word of this file (bit 1: tokens appended past the capacity).
__device__ unsigned int g_ris_cache4_error;

namespace {

template <typename T>
__device__ __forceinline__ float to_f(T x);
template <>
__device__ __forceinline__ float to_f<float>(float x) { return x; }
template <>
__device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }

// x[0 .. N-1], N elements in a row, N * sizeof(T) a multiple of 4 and the address aligned to it (up to 16)
template <typename T, int N>
__device__ __forceinline__ void load_row(const T *p, float *x)
{
    constexpr int B = N * (int)sizeof(T), W = B >= 16 ? 16 : B;
    uint32_t w[B / 4];
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
#pragma unroll
    for (int e = 0; e < N; ++e) {
        if constexpr (sizeof(T) == 4)
            x[e] = __uint_as_float(w[e]);
        else
            x[e] = __uint_as_float((e & 1) ? (w[e >> 1] & 0xFFFF0000u) : (w[e >> 1] << 16));
    }
}

// |x| for a maximum that a NaN or an infinity must win: the bits without the sign
__device__ __forceinline__ uint32_t mag(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// The scale of a group whose largest magnitude has these bits; NaN where a value is not finite, so that
// the row then stands for NaN and no other row is touched
__device__ __forceinline__ __nv_bfloat16 scale_of(uint32_t top)
{
    return __float2bfloat16_rn(top >= 0x7F800000u ? __uint_as_float(0x7FFFFFFFu) : __uint_as_float(top) * (1.f / 6.f));
}

// the codes of a and b (a in the low half)
__device__ __forceinline__ uint32_t code2(float a, float b, float s)
{
    const float x = s > 0.f ? __fdiv_rn(a, s) : 0.f, y = s > 0.f ? __fdiv_rn(b, s) : 0.f;
    uint16_t r;
    asm("{\n\t.reg .b8 t;\n\tcvt.rn.satfinite.e2m1x2.f32 t, %1, %2;\n\tcvt.u16.u8 %0, t;\n\t}" : "=h"(r) : "f"(y), "f"(x));
    return r;
}

constexpr int kAppendThreads = 256;

// blockIdx.y 0: keys, four lanes to a row; 1: values, eight lanes to a row. Each lane loads what it
// stores, so rows are read and written in whole sectors; a group's maximum comes from its lanes by
// shuffles. Bound by HBM: a row is read once (2 D bytes of bf16) and D / 2 + D / 16 bytes are written.
template <typename T, int D>
__global__ void __launch_bounds__(kAppendThreads) k_cache4_append(const Cache4AppendArgs a)
{
    constexpr int NG = D / kCacheGroup;
    const bool values = blockIdx.y != 0;
    const int lanes = values ? 8 : 4, u = threadIdx.x & (lanes - 1);
    const int64_t r = (int64_t)blockIdx.x * (kAppendThreads / lanes) + threadIdx.x / lanes;  // token and head
    const int64_t n_rows = a.total * a.c.Hkv;
    const bool in = r < n_rows;
    const int64_t tok = (in ? r : n_rows - 1) / a.c.Hkv;
    const int head = (int)((in ? r : n_rows - 1) - tok * a.c.Hkv);
    const int b = a.seq_of[tok], i = (int)tok - a.off[b];
    const int64_t slot = (int64_t)(a.start != nullptr ? a.start[b] : a.c.length[b]) + i;
    const bool ok = slot >= 0 && slot < a.c.cap;
    if (in && !ok) atomicOr(&g_ris_cache4_error, 2u);
    const int64_t row = ((int64_t)b * a.c.Hkv + head) * a.c.cap + slot;
    if (!values) {
        float x[NG][8];
        const T *p = reinterpret_cast<const T *>(a.k) + tok * a.k_stride + head * D + 8 * u;
#pragma unroll
        for (int g = 0; g < NG; ++g) load_row<T, 8>(p + kCacheGroup * g, x[g]);
        uint32_t w[NG], sc[NG];
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, mag(x[g][e]));
            top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
            top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
            const __nv_bfloat16 s = scale_of(top);
            sc[g] = __bfloat16_as_ushort(s);
            const float sf = __bfloat162float(s);
            w[g] = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) w[g] |= code2(x[g][2 * e], x[g][2 * e + 1], sf) << (8 * e);
        }
        if (in && ok) {
            uint8_t *dst = a.c.k + row * (D / 2) + u * (4 * NG);
            if constexpr (NG == 4)
                *reinterpret_cast<uint4 *>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
            else
                *reinterpret_cast<uint2 *>(dst) = make_uint2(w[0], w[1]);
            if (u == 0) {
                uint32_t *ds = reinterpret_cast<uint32_t *>(a.c.k_scale + row * NG);
#pragma unroll
                for (int g = 0; g < NG / 2; ++g) ds[g] = sc[2 * g] | (sc[2 * g + 1] << 16);
            } else if (u == 1) {
                a.c.pos[row] = a.positions[tok];
            } else if (u == 2) {
                a.c.weight[row] = a.weight != nullptr ? a.weight[(int64_t)head * a.total + tok] : 0.f;
            }
        }
    } else {
        constexpr int NM = D / 16;
        float x[NM][2];
        const T *p = reinterpret_cast<const T *>(a.v) + tok * a.v_stride + head * D + 2 * u;
#pragma unroll
        for (int m = 0; m < NM; ++m) load_row<T, 2>(p + 16 * m, x[m]);
        uint32_t w[NM / 4] = {}, sc[NG];
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            uint32_t top = max(max(mag(x[2 * g][0]), mag(x[2 * g][1])), max(mag(x[2 * g + 1][0]), mag(x[2 * g + 1][1])));
#pragma unroll
            for (int o = 1; o < 8; o <<= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
            const __nv_bfloat16 s = scale_of(top);
            sc[g] = __bfloat16_as_ushort(s);
            const float sf = __bfloat162float(s);
#pragma unroll
            for (int e = 2 * g; e < 2 * g + 2; ++e) w[e / 4] |= code2(x[e][0], x[e][1], sf) << (8 * (e & 3));
        }
        if (in && ok) {
            uint8_t *dst = a.c.v + row * (D / 2) + u * NM;
            if constexpr (NM == 8)
                *reinterpret_cast<uint2 *>(dst) = make_uint2(w[0], w[1]);
            else
                *reinterpret_cast<uint32_t *>(dst) = w[0];
            if (u == 0) {
                uint32_t *ds = reinterpret_cast<uint32_t *>(a.c.v_scale + row * NG);
#pragma unroll
                for (int g = 0; g < NG / 2; ++g) ds[g] = sc[2 * g] | (sc[2 * g + 1] << 16);
            }
        }
    }
    // the new lengths: written at once where the rows start at given slots, else by the last CTA,
    // once every CTA has read the old ones
    bool last = a.start != nullptr && blockIdx.x == 0 && blockIdx.y == 0;
    if (a.start == nullptr) {
        __shared__ bool done;
        __syncthreads();
        if (threadIdx.x == 0) {
            __threadfence();
            done = atomicAdd(a.ticket, 1u) == gridDim.x * gridDim.y - 1;
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

// the two values of a byte
__device__ __forceinline__ __half2 values2(uint32_t byte)
{
    uint32_t r;
    asm("{\n\t.reg .b8 t, z0, z1, z2;\n\tmov.b32 {t, z0, z1, z2}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, t;\n\t}" : "=r"(r) : "r"(byte));
    return *reinterpret_cast<const __half2 *>(&r);
}

// One thread per four elements of a row of the output: two bytes in, 16 bytes out. Bound by the fp32
// rows that it writes.
constexpr int kReadThreads = 256;
template <int D>
__global__ void __launch_bounds__(kReadThreads) k_cache4_read(const Cache4Args c, const int32_t *first, int64_t count, float *ko,
                                                              float *vo)
{
    constexpr int Q = D / 4, NG = D / kCacheGroup, NM = D / 16;
    const int64_t t = (int64_t)blockIdx.x * kReadThreads + threadIdx.x;
    const int64_t n = (int64_t)c.B * c.Hkv * count * Q;
    if (t >= n) return;
    const int e = (int)(t % Q);  // elements 4 e .. 4 e + 3: bytes 2 e, 2 e + 1 in natural order
    const int64_t r = t / Q, bh = r / count, i = r % count;
    const int b = (int)(bh / c.Hkv);
    const int64_t slot = i + (first != nullptr ? first[b] : 0);
    const bool there = slot >= 0 && slot < min((int64_t)c.length[b], c.cap);
    const bool values = blockIdx.y != 0;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    if (there) {
        const int64_t row = bh * c.cap + slot;
        uint32_t b0, b1;
        if (!values) {
            const int word = e / 2;  // 8 elements
            const uint8_t *p = c.k + row * (D / 2) + ((word & 3) * NG + (word >> 2)) * 4 + (e & 1) * 2;
            const uint32_t w = *reinterpret_cast<const uint16_t *>(p);
            b0 = w & 0xFFu, b1 = w >> 8;
        } else {
            const int tile = e / 4, col = 2 * (e & 3);
            const uint8_t *p = c.v + row * (D / 2) + tile;
            b0 = p[col * NM], b1 = p[(col + 1) * NM];
        }
        const uint32_t s = (values ? c.v_scale : c.k_scale)[row * NG + e / 8];
        const float sf = __uint_as_float(s << 16);
        const float2 lo = __half22float2(values2(b0)), hi = __half22float2(values2(b1));
        x = make_float4(lo.x * sf, lo.y * sf, hi.x * sf, hi.y * sf);
    }
    reinterpret_cast<float4 *>(values ? vo : ko)[t] = x;
}

// ---------------------------------------------------------------- attention of one token
constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kTile = 16;                      // slots of a warp's product
constexpr int kWarpTiles = 4;                  // tiles of a warp in a stage
constexpr int kStageSlots = kWarps * kWarpTiles * kTile;  // 256
constexpr int kStages = 2;
constexpr int kMinExp = -114;                  // smallest exponent of a value scale that counts as such

template <int D>
struct Lay {
    static constexpr int NG = D / kCacheGroup, NM = D / 16;
    static constexpr int CODES = D / 2, SCALES = 2 * NG;  // bytes of a slot
    static constexpr int OFF_K = 0, OFF_V = OFF_K + kStageSlots * CODES, OFF_KS = OFF_V + kStageSlots * CODES,
                         OFF_VS = OFF_KS + kStageSlots * SCALES, STAGE = OFF_VS + kStageSlots * SCALES;
    static constexpr int OFF_BARS = kStages * STAGE, BYTES = OFF_BARS + 8 * kStages;
};

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity)
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
        if (clock64() - t0 > (1LL << 31)) return false;
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
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
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
__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
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
__device__ __forceinline__ float bf16_at(uint32_t w, int e) { return __uint_as_float((e & 1) ? (w & 0xFFFF0000u) : (w << 16)); }

// Slot of row r (0 .. 15) of a tile: the rows that a lane needs as pairs along the product's inner
// dimension, 2 t, 2 t + 1, 2 t + 8 and 2 t + 9, are slots t, 4 + t, 8 + t and 12 + t, so that the four lanes t read
// neighbouring rows of the values.
__device__ __forceinline__ int tile_slot(int r) { return ((r & 7) >> 1) + 4 * (r & 1) + (r & 8); }

// One CTA per (range of slots, KV head, sequence). Its four warps take tiles of 16 slots in turn, each with
// a softmax of its own over the slots that it saw; bulk copies bring stages of 256 slots (codes and
// scales, contiguous per KV head) into a ring of two. A tile:
//   S^T = K q^T  rows are slots, columns up to 8 query heads: the codes as fp16 (exact) straight from
//                the lane's word, one accumulator per group of 32, which the group's scale then multiplies in
//                fp32 (so the products are exact up to fp32 sums); the query as fp16 scaled by a power of two, with a second fp16 of
//                what that leaves for fp32 inputs;
//   O^T += V^T P^T  the weights times the slot's scale, per group of 32, as fp16 scaled by 2^12 over the
//                largest scale so far (a weight of 2^-26 of the largest is still normal), transposed by movmatrix; with SPLIT a second fp16
//                of what the first leaves, for fp32 outputs; values as fp16 pairs of slots by byte permutes.
// Slots past the length enter with score -infinity and scale 0, whatever lies there.
// G query heads of a KV head: 8 of them per product; QB products of a CTA share the unpacked codes' loads.
template <typename T, bool SPLIT, int D, int QB>
__global__ void __launch_bounds__(kThreads) k_cache4_attend(const Cache4AttendArgs a)
{
    using L = Lay<D>;
    constexpr int NG = L::NG, NM = L::NM;
    constexpr bool LO = sizeof(T) == 4;  // the query needs a second part
    extern __shared__ __align__(128) unsigned char smem[];
    const uint32_t sbase = smem_u32(smem);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g8 = lane >> 2, t4 = lane & 3;
    const int b = blockIdx.z, kvh = blockIdx.y % a.c.Hkv, h0 = blockIdx.y / a.c.Hkv * (8 * QB);  // first head of the group
    const int nh = min(8 * QB, a.G - h0);
    const int64_t len = max(0, min(a.c.length[b], (int)min(a.reach, (int64_t)INT32_MAX)));
    const int64_t first = (int64_t)blockIdx.x * a.chunk;
    const int n = (int)max((int64_t)0, min((int64_t)a.chunk, len - first));  // slots of this CTA
    const int64_t head0 = (int64_t)b * a.Hq + kvh * a.G + h0;                 // its first query head
    if (n == 0 && blockIdx.x != 0) return;
    const int64_t row0 = ((int64_t)b * a.c.Hkv + kvh) * a.c.cap + first;
    const int n_stages = (n + kStageSlots - 1) / kStageSlots;
    auto fetch = [&](int st) {  // by one thread
        const int s0 = st * kStageSlots, rows = min(kStageSlots, (n - s0 + 15) / 16 * 16);
        const uint32_t bar = sbase + L::OFF_BARS + 8 * (st % kStages), dst = sbase + st % kStages * L::STAGE;
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(rows * 2 * (L::CODES + L::SCALES))
                     : "memory");
        bulk_load(dst + L::OFF_K, a.c.k + (row0 + s0) * L::CODES, rows * L::CODES, bar);
        bulk_load(dst + L::OFF_KS, a.c.k_scale + (row0 + s0) * NG, rows * L::SCALES, bar);
        bulk_load(dst + L::OFF_V, a.c.v + (row0 + s0) * L::CODES, rows * L::CODES, bar);
        bulk_load(dst + L::OFF_VS, a.c.v_scale + (row0 + s0) * NG, rows * L::SCALES, bar);
    };
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i)
            asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(sbase + L::OFF_BARS + 8 * i) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        for (int st = 0; st < min(kStages, n_stages); ++st) fetch(st);
    }
    // the queries: lane (g8, t4) holds elements 32 g + 8 t4 .. + 7 of head g8 of each block, scaled by 2^-e
    uint32_t qh[QB][NG][4], ql[LO ? QB : 1][LO ? NG : 1][4];
    float unscale[QB][2];  // of heads 2 t4, 2 t4 + 1: log2(e) / sqrt(D) 2^e
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const int h = 8 * qb + g8;
        const bool have = h < nh;
        const T *q = reinterpret_cast<const T *>(a.q) + (head0 + (have ? h : 0)) * D + 8 * t4;
        float x[NG][8];
        uint32_t top = 0;
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            load_row<T, 8>(q + kCacheGroup * g, x[g]);
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, mag(x[g][e]));
        }
        top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
        top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
        // |q| 2^-e below 2^13; the exponent stays where both factors are normal numbers
        const int e2 = min(max((int)(top >> 23) - 127 - 12, -100), 100);
        const float down = pow2i(-e2), up = have ? pow2i(e2) * a.scale_log2 : 0.f;
#pragma unroll
        for (int g = 0; g < NG; ++g)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float u = have ? x[g][2 * e] * down : 0.f, v = have ? x[g][2 * e + 1] * down : 0.f;
                qh[qb][g][e] = pack_half(u, v);
                if constexpr (LO) ql[qb][g][e] = pack_rest(u, v, qh[qb][g][e]);
            }
        unscale[qb][0] = __shfl_sync(0xFFFFFFFFu, up, 8 * t4);
        unscale[qb][1] = __shfl_sync(0xFFFFFFFFu, up, 8 * t4 + 4);
    }
    float m[QB][2], l[QB][2], o[QB][NM][4];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        m[qb][0] = m[qb][1] = -INFINITY;
        l[qb][0] = l[qb][1] = 0.f;
#pragma unroll
        for (int e = 0; e < NM; ++e) o[qb][e][0] = o[qb][e][1] = o[qb][e][2] = o[qb][e][3] = 0.f;
    }
    int ev = kMinExp;  // O is in units of 2^(ev - 12), ev the exponent of the largest value scale so far
    bool ok = true;
    __syncthreads();
    for (int st = 0; st < n_stages; ++st) {
        // (a warp whose wait gave up only skips the work: every warp meets the others at each barrier)
        if (ok) ok = mbar_wait(sbase + L::OFF_BARS + 8 * (st % kStages), (st / kStages) & 1);
        const unsigned char *sm = smem + st % kStages * L::STAGE;
        const int s0 = st * kStageSlots, ns = min(kStageSlots, n - s0);  // slots of the stage
        const int n_tiles = (ns + kTile - 1) / kTile;
        if (ok && warp < n_tiles) {
            // the value scales of this lane's slots, and the largest of the warp's
            uint32_t vsc[kWarpTiles][2][NG / 2], top = 0;
#pragma unroll
            for (int i = 0; i < kWarpTiles; ++i)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const int slot = (warp + kWarps * i) * kTile + tile_slot(g8 + 8 * r);
                    const bool there = slot < ns;
                    const uint32_t *p = reinterpret_cast<const uint32_t *>(sm + L::OFF_VS + (there ? slot : 0) * L::SCALES);
#pragma unroll
                    for (int g = 0; g < NG / 2; ++g) {
                        vsc[i][r][g] = there ? p[g] : 0u;
                        top = __vmaxu2(top, vsc[i][r][g]);
                    }
                }
            top = max(top & 0xFFFFu, top >> 16);
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, x));
            const int e_new = max(ev, min((int)(top >> 7) - 127, 127));
            const float ov = e_new - ev > 126 ? 0.f : pow2i(ev - e_new);  // O in the new units
            ev = e_new;
            const float to16 = pow2i(12 - ev);
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) {
                float s[kWarpTiles][4];
#pragma unroll
                for (int i = 0; i < kWarpTiles; ++i) {
                    const int tile = warp + kWarps * i;
                    if (tile >= n_tiles) {
                        s[i][0] = s[i][1] = s[i][2] = s[i][3] = -INFINITY;
                        continue;
                    }
                    uint32_t kw[2][NG];
                    float ks[2][NG];
                    bool there[2];
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const int slot = tile * kTile + tile_slot(g8 + 8 * r);
                        there[r] = slot < ns;
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
                        for (int g = 0; g < NG; ++g) ks[r][g] = bf16_at(ps[g / 2], g);
                    }
                    float acc[4] = {};
#pragma unroll
                    for (int g = 0; g < NG; ++g) {
                        uint32_t x[4], y[4];
                        unpack4(kw[0][g], x);
                        unpack4(kw[1][g], y);
                        float d[4] = {};
                        const uint32_t f0[4] = {x[0], y[0], x[1], y[1]}, f1[4] = {x[2], y[2], x[3], y[3]};
                        mma(d, f0, qh[qb][g][0], qh[qb][g][1]);
                        mma(d, f1, qh[qb][g][2], qh[qb][g][3]);
                        if constexpr (LO) {
                            mma(d, f0, ql[qb][g][0], ql[qb][g][1]);
                            mma(d, f1, ql[qb][g][2], ql[qb][g][3]);
                        }
                        acc[0] = fmaf(d[0], ks[0][g], acc[0]);
                        acc[1] = fmaf(d[1], ks[0][g], acc[1]);
                        acc[2] = fmaf(d[2], ks[1][g], acc[2]);
                        acc[3] = fmaf(d[3], ks[1][g], acc[3]);
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[i][e] = there[e >> 1] ? acc[e] * unscale[qb][e & 1] : -INFINITY;
                    if (a.scores != nullptr) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int h = 8 * qb + 2 * t4 + (e & 1);
                            if (there[e >> 1] && h < nh)
                                a.scores[(head0 + h) * a.c.cap + first + s0 + tile * kTile + tile_slot(g8 + 8 * (e >> 1))] = s[i][e];
                        }
                    }
                }
                float nm[2], al[2], ref[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float x = fmaxf(s[0][e], s[0][e + 2]);
#pragma unroll
                    for (int i = 1; i < kWarpTiles; ++i) x = fmaxf(x, fmaxf(s[i][e], s[i][e + 2]));
#pragma unroll
                    for (int y = 4; y < 32; y <<= 1) x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, y));
                    nm[e] = fmaxf(m[qb][e], x);
                    ref[e] = nm[e] == -INFINITY ? 0.f : nm[e];
                    al[e] = ex2(m[qb][e] - ref[e]);
                    m[qb][e] = nm[e];
                    l[qb][e] *= al[e];
                }
                // fp32 outputs: the stage's products from zero, added to O in fp32 afterwards. (The tensor pipe's
                // additions cut off: over thousands of slots in one accumulator 2e-6 of the result.)
                float part[SPLIT ? NM : 1][4] = {};
                if constexpr (!SPLIT) {
#pragma unroll
                    for (int e = 0; e < NM; ++e)
#pragma unroll
                        for (int c = 0; c < 4; ++c) o[qb][e][c] *= al[c & 1] * ov;
                }
#pragma unroll
                for (int i = 0; i < kWarpTiles; ++i) {
                    const int tile = warp + kWarps * i;
                    if (tile >= n_tiles) continue;
                    float p[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        p[e] = ex2(s[i][e] - ref[e & 1]);
                        l[qb][e & 1] += p[e];
                        p[e] *= to16;
                    }
                    uint32_t bh[NG][2], bl[SPLIT ? NG : 1][2];
#pragma unroll
                    for (int g = 0; g < NG; ++g)
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            const float sc = bf16_at(vsc[i][r][g / 2], g);
                            const float x = p[2 * r] * sc, y = p[2 * r + 1] * sc;
                            const uint32_t hi = pack_half(x, y);
                            if constexpr (SPLIT) bl[g][r] = transpose8(pack_rest(x, y, hi));
                            bh[g][r] = transpose8(hi);
                        }
                    uint32_t vw[4][NM / 4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const unsigned char *p8 = sm + L::OFF_V + (tile * kTile + 4 * r + t4) * L::CODES + g8 * NM;
                        if constexpr (NM == 8) {
                            const uint2 w = *reinterpret_cast<const uint2 *>(p8);
                            vw[r][0] = w.x, vw[r][1] = w.y;
                        } else {
                            vw[r][0] = *reinterpret_cast<const uint32_t *>(p8);
                        }
                    }
#pragma unroll
                    for (int q4 = 0; q4 < NM / 4; ++q4) {
                        uint32_t x[4][4];
#pragma unroll
                        for (int r = 0; r < 4; ++r) unpack4(vw[r][q4], x[r]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int tl = 4 * q4 + e;
                            const uint32_t f[4] = {__byte_perm(x[0][e], x[1][e], 0x5410), __byte_perm(x[0][e], x[1][e], 0x7632),
                                                   __byte_perm(x[2][e], x[3][e], 0x5410), __byte_perm(x[2][e], x[3][e], 0x7632)};
                            if constexpr (SPLIT) {
                                mma(part[tl], f, bl[tl / 2][0], bl[tl / 2][1]);
                                mma(part[tl], f, bh[tl / 2][0], bh[tl / 2][1]);
                            } else {
                                mma(o[qb][tl], f, bh[tl / 2][0], bh[tl / 2][1]);
                            }
                        }
                    }
                }
                if constexpr (SPLIT) {
#pragma unroll
                    for (int e = 0; e < NM; ++e)
#pragma unroll
                        for (int c = 0; c < 4; ++c) o[qb][e][c] = fmaf(o[qb][e][c], al[c & 1] * ov, part[e][c]);
                }
            }
        }
        __syncthreads();  // every warp is done with the stage
        if (threadIdx.x == 0 && ok && st + kStages < n_stages) fetch(st + kStages);
    }
    ok = __syncthreads_and(ok);
    if (!ok) {  // (a copy that never landed: the outputs are undefined)
        if (threadIdx.x == 0) atomicOr(&g_ris_cache4_error, 4u);
        return;
    }
    // the four warps' parts of each head, through shared memory: [warp][head][D] and (maximum, sum)
    float *const so = reinterpret_cast<float *>(smem);
    float2 *const sml = reinterpret_cast<float2 *>(smem + kWarps * 8 * QB * D * 4);
    const float back = pow2i(ev - 12);
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float x = l[qb][e];
#pragma unroll
            for (int y = 4; y < 32; y <<= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, y);
            const int h = 8 * qb + 2 * t4 + e;
            if (g8 == 0) sml[warp * 8 * QB + h] = make_float2(m[qb][e], x);
#pragma unroll
            for (int tl = 0; tl < NM; ++tl)
                *reinterpret_cast<float2 *>(so + (warp * 8 * QB + h) * D + 16 * tl + 2 * g8) =
                    make_float2(o[qb][tl][e] * back, o[qb][tl][e + 2] * back);
        }
    }
    __syncthreads();
    for (int t = threadIdx.x; t < nh * D; t += kThreads) {
        const int h = t / D, d = t % D;
        float M = -INFINITY, sum = 0.f, x = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) M = fmaxf(M, sml[w * 8 * QB + h].x);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float2 ml = sml[w * 8 * QB + h];
            const float f = ml.x == -INFINITY ? 0.f : exp2f(ml.x - M);
            sum = fmaf(ml.y, f, sum);
            x = fmaf(so[(w * 8 * QB + h) * D + d], f, x);
        }
        const int64_t part = (head0 + h) * a.n_chunks + blockIdx.x;
        a.part_o[part * D + d] = x;
        if (d == 0) a.part_ml[part] = make_float2(M, sum);
    }
}

// Joins the ranges of a sequence: one CTA per (query head, sequence), a thread per channel; then
// (weights) CTAs that add up what each slot got from the heads of its KV head, from the scores that the first kernel left.
constexpr int kJoinThreads = 128;
constexpr int kWeightSlots = 1024;  // slots of a CTA

template <typename TO, int D>
__global__ void __launch_bounds__(kJoinThreads) k_cache4_join(const Cache4AttendArgs a)
{
    const int b = blockIdx.z;
    const int64_t len = max(0, min(a.c.length[b], (int)min(a.reach, (int64_t)INT32_MAX)));
    const int na = max(1, (int)((len + a.chunk - 1) / a.chunk));  // ranges that hold slots
    if ((int)blockIdx.x < a.Hq) {
        const int64_t h = (int64_t)b * a.Hq + blockIdx.x;
        const float2 *ml = a.part_ml + h * a.n_chunks;
        float M = -INFINITY, sum = 0.f, x = 0.f;
        for (int i = 0; i < na; ++i) M = fmaxf(M, ml[i].x);
        const int d = threadIdx.x;
        if (d < D) {
            const float *po = a.part_o + h * a.n_chunks * D + d;
#pragma unroll 8
            for (int i = 0; i < na; ++i) {
                const float2 y = ml[i];
                const float f = y.x == -INFINITY ? 0.f : exp2f(y.x - M);
                sum = fmaf(y.y, f, sum);
                x = fmaf(po[(int64_t)i * D], f, x);
            }
            x = sum == 0.f ? 0.f : x / sum;  // no slot: zeros
            if constexpr (sizeof(TO) == 4)
                reinterpret_cast<float *>(a.out)[h * D + d] = x;
            else
                reinterpret_cast<__nv_bfloat16 *>(a.out)[h * D + d] = __float2bfloat16_rn(x);
            if (d == 0 && a.lse != nullptr) a.lse[h] = (M + log2f(sum)) * kLn2;
        }
        return;
    }
    // weights
    const int w = blockIdx.x - a.Hq, blocks = (gridDim.x - a.Hq) / a.c.Hkv, kvh = w / blocks;
    const int64_t s0 = (int64_t)(w % blocks) * kWeightSlots;
    if (s0 >= len) return;
    extern __shared__ float2 stat[];  // [G]
    for (int h = threadIdx.x; h < a.G; h += kJoinThreads) {
        const float2 *ml = a.part_ml + ((int64_t)b * a.Hq + kvh * a.G + h) * a.n_chunks;
        float M = -INFINITY, sum = 0.f;
        for (int i = 0; i < na; ++i) M = fmaxf(M, ml[i].x);
        for (int i = 0; i < na; ++i) sum = fmaf(ml[i].y, exp2f(ml[i].x - M), sum);
        stat[h] = make_float2(M, 1.f / sum);
    }
    __syncthreads();
    const int64_t row = ((int64_t)b * a.c.Hkv + kvh) * a.c.cap;
    const float *sc = a.scores + ((int64_t)b * a.Hq + kvh * a.G) * a.c.cap;
    for (int64_t s = s0 + threadIdx.x; s < min(s0 + kWeightSlots, len); s += kJoinThreads) {
        float x = 0.f;
        for (int h = 0; h < a.G; ++h) x = fmaf(ex2(sc[h * a.c.cap + s] - stat[h].x), stat[h].y, x);
        a.weight_out[row + s] = (a.weight_in != nullptr ? a.weight_in[row + s] : 0.f) + x;
    }
}

template <typename T, bool SPLIT, int D, int QB>
cudaError_t launch_part(const Cache4AttendArgs &a, cudaStream_t s)
{
    auto kern = k_cache4_attend<T, SPLIT, D, QB>;
    constexpr int bytes = std::max(Lay<D>::BYTES, kWarps * 8 * QB * (D * 4 + 8));
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != cudaSuccess) return e;
    const int blocks = (a.G + 8 * QB - 1) / (8 * QB);
    kern<<<dim3((unsigned)a.n_chunks, (unsigned)(a.c.Hkv * blocks), (unsigned)a.c.B), kThreads, bytes, s>>>(a);
    note_launch();
    return cudaGetLastError();
}
template <typename T, bool SPLIT>
cudaError_t launch_part_d(const Cache4AttendArgs &a, cudaStream_t s)
{
    if (a.G > 8) return a.c.D == 128 ? launch_part<T, SPLIT, 128, 2>(a, s) : launch_part<T, SPLIT, 64, 2>(a, s);
    return a.c.D == 128 ? launch_part<T, SPLIT, 128, 1>(a, s) : launch_part<T, SPLIT, 64, 1>(a, s);
}
template <typename TO>
cudaError_t launch_join(const Cache4AttendArgs &a, cudaStream_t s)
{
    const int64_t blocks = a.weight_out != nullptr ? (a.reach + kWeightSlots - 1) / kWeightSlots * a.c.Hkv : 0;
    const dim3 grid((unsigned)(a.Hq + blocks), 1, (unsigned)a.c.B);
    const size_t bytes = a.weight_out != nullptr ? a.G * sizeof(float2) : 0;
    if (a.c.D == 128)
        k_cache4_join<TO, 128><<<grid, kJoinThreads, bytes, s>>>(a);
    else
        k_cache4_join<TO, 64><<<grid, kJoinThreads, bytes, s>>>(a);
    note_launch();
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_cache4_append(const Cache4AppendArgs &a, int dtype, cudaStream_t s)
{
    const int64_t rows = a.total * a.c.Hkv, per = kAppendThreads / 8;
    const dim3 grid((unsigned)((rows + per - 1) / per), 2);
    if (dtype == RIS_F32) {
        if (a.c.D == 128)
            k_cache4_append<float, 128><<<grid, kAppendThreads, 0, s>>>(a);
        else
            k_cache4_append<float, 64><<<grid, kAppendThreads, 0, s>>>(a);
    } else {
        if (a.c.D == 128)
            k_cache4_append<__nv_bfloat16, 128><<<grid, kAppendThreads, 0, s>>>(a);
        else
            k_cache4_append<__nv_bfloat16, 64><<<grid, kAppendThreads, 0, s>>>(a);
    }
    note_launch();
    return cudaGetLastError();
}

cudaError_t launch_cache4_read(const Cache4Args &c, const int32_t *first, int64_t count, float *k, float *v, cudaStream_t s)
{
    const int64_t n = (int64_t)c.B * c.Hkv * count * (c.D / 4);
    const dim3 grid((unsigned)((n + kReadThreads - 1) / kReadThreads), 2);
    if (c.D == 128)
        k_cache4_read<128><<<grid, kReadThreads, 0, s>>>(c, first, count, k, v);
    else
        k_cache4_read<64><<<grid, kReadThreads, 0, s>>>(c, first, count, k, v);
    note_launch();
    return cudaGetLastError();
}

cudaError_t launch_cache4_attend(const Cache4AttendArgs &a, int dtype, int out_dtype, cudaStream_t s)
{
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

unsigned int read_cache4_error()
{
    unsigned int v = 0, zero = 0;
    if (cudaMemcpyFromSymbol(&v, g_ris_cache4_error, sizeof(v)) != cudaSuccess) return 0;
    if (v != 0) cudaMemcpyToSymbol(g_ris_cache4_error, &zero, sizeof(zero));
    return v;
}

}  // namespace ris
