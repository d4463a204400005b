// Causal attention over packed prompts on the FP32 pipe: fp32 inputs, which never pass through a
// narrower product, and the weight that each key got from a sequence's last rows.
//
// k_packed_f32: one CTA per (64 query rows, query head) walks the keys in tiles of 64 with a running
// maximum and sum: S = Q K^T with a 4 x 4 patch per thread (Q and K d-major in shared memory), the softmax
// over the 16 lanes that share a row, P d-major over the keys' place, O += P V with a 4 x D/16 patch in registers.
// Bound by the FMA pipe (4 D flops per pair and head); per step of d a warp reads 3 wavefronts of shared
// memory for 16 packed multiply-adds, so both pipes are near even.
//
// k_packed_weights: one thread per key holds the key's row in registers and walks the last rows of the
// group's heads, broadcast from shared memory: w_j = sum_i,h exp2(s_ij - m_i) / l_i.
#include <cuda_bf16.h>

#include <cstdint>
#include <type_traits>

#include "attn_common.cuh"
#include "serve.h"

namespace ris {
namespace {

constexpr int BM = 64, BN = 64, LD = BM + 4;  // rows and keys of a tile, pitch of the d-major arrays
constexpr int kThreads = 256;
constexpr int kHalves = kPackRows / BM;

__device__ __forceinline__ float4 load4(const float *p) { return *reinterpret_cast<const float4 *>(p); }
__device__ __forceinline__ void store4(float *p, float4 x) { *reinterpret_cast<float4 *>(p) = x; }
__device__ __forceinline__ void store4(__nv_bfloat16 *p, float4 x)
{
    const __nv_bfloat162 a = __floats2bfloat162_rn(x.x, x.y), b = __floats2bfloat162_rn(x.z, x.w);
    *reinterpret_cast<uint2 *>(p) =
        make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
}

__device__ __forceinline__ uint64_t f2(float x, float y)
{
    uint64_t d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(x), "f"(y));
    return d;
}
__device__ __forceinline__ uint64_t f2_fma(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t f2_mul(uint64_t a, uint64_t b)
{
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ float2 f2_get(uint64_t v)
{
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}

// x[row][d] of up to 64 rows of one head, d-major into dst[d][row]; rows past `rows` as zeros
template <int D>
__device__ __forceinline__ void stage_t(float *dst, const float *x, int64_t stride, int rows)
{
    for (int t = threadIdx.x; t < BM * (D / 4); t += kThreads) {
        const int r = t % BM, d = t / BM * 4;
        const float4 v = r < rows ? load4(x + r * stride + d) : make_float4(0.f, 0.f, 0.f, 0.f);
        dst[d * LD + r] = v.x;
        dst[(d + 1) * LD + r] = v.y;
        dst[(d + 2) * LD + r] = v.z;
        dst[(d + 3) * LD + r] = v.w;
    }
}

template <typename TO, int D>
__global__ void __launch_bounds__(kThreads, 2) k_packed_f32(const PackedArgs a)
{
    extern __shared__ __align__(16) float sm[];
    float *const qs = sm, *const ks = qs + D * LD, *const vs = ks + D * LD, *const ps = ks;
    const int b = blockIdx.x, h = b % a.Hq, part = b / a.Hq % kHalves;
    const PackItem it = a.items[b / a.Hq / kHalves];
    const int r0 = it.row + part * BM, rows = min(BM, it.q_len - r0);
    if (rows <= 0) return;
    const int g = h / a.G;
    const int shift = it.k_len - it.q_len;              // row i sees keys j <= i + shift
    const int keys = max(0, min(it.k_len, r0 + rows + shift));  // that the last of the rows sees
    const float *q = reinterpret_cast<const float *>(a.q) + (int64_t)(it.q_base + r0) * a.q_stride + h * D;
    const float *k = reinterpret_cast<const float *>(a.k) + (int64_t)it.k_base * a.k_stride + g * D;
    const float *v = reinterpret_cast<const float *>(a.v) + (int64_t)it.k_base * a.v_stride + g * D;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    stage_t<D>(qs, q, a.q_stride, rows);
    constexpr int C = D / 16;  // columns of O of a thread: 4 tx + 64 x ..
    uint64_t o[4][C / 2] = {};
    float m[4], l[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) m[i] = -INFINITY, l[i] = 0.f;
    for (int k0 = 0; k0 < keys; k0 += BN) {
        const int kn = min(BN, keys - k0);
        __syncthreads();  // the tiles of the last step are done with
        stage_t<D>(ks, k + (int64_t)k0 * a.k_stride, a.k_stride, kn);
        for (int t = threadIdx.x; t < BN * (D / 4); t += kThreads) {
            const int r = t / (D / 4), d = t % (D / 4) * 4;
            // a key that is not there weighs nothing, whatever lies in its place
            store4(vs + r * D + d, r < kn ? load4(v + (int64_t)(k0 + r) * a.v_stride + d) : make_float4(0.f, 0.f, 0.f, 0.f));
        }
        __syncthreads();
        uint64_t s2[4][2] = {};
#pragma unroll 8
        for (int d = 0; d < D; ++d) {
            const float4 qa = *reinterpret_cast<const float4 *>(qs + d * LD + 4 * ty);
            const ulonglong2 kb = *reinterpret_cast<const ulonglong2 *>(ks + d * LD + 4 * tx);
            const float qr[4] = {qa.x, qa.y, qa.z, qa.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint64_t qq = f2(qr[i], qr[i]);
                s2[i][0] = f2_fma(qq, kb.x, s2[i][0]);
                s2[i][1] = f2_fma(qq, kb.y, s2[i][1]);
            }
        }
        __syncthreads();  // the keys' place takes P
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 lo = f2_get(s2[i][0]), hi = f2_get(s2[i][1]);
            float s[4] = {lo.x, lo.y, hi.x, hi.y};
            const int last = r0 + 4 * ty + i + shift - k0 - 4 * tx;  // last key of the patch that the row sees
            float mx = -INFINITY;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[e] = e <= last && 4 * tx + e < kn ? s[e] * a.scale_log2 : -INFINITY;
                mx = fmaxf(mx, s[e]);
            }
#pragma unroll
            for (int x = 8; x > 0; x >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, x));
            const float nm = fmaxf(m[i], mx), ref = nm == -INFINITY ? 0.f : nm;
            const float al = exp2f(m[i] - ref);
            m[i] = nm;
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[e] = exp2f(s[e] - ref);
                sum += s[e];
                ps[(4 * tx + e) * LD + 4 * ty + i] = s[e];
            }
            l[i] = fmaf(l[i], al, sum);  // this lane's part of the row's sum
            const uint64_t al2 = f2(al, al);
#pragma unroll
            for (int c = 0; c < C / 2; ++c) o[i][c] = f2_mul(o[i][c], al2);
        }
        __syncthreads();
        // O += P V; where some row does not see the whole tile, a row takes only the keys that it sees (0 times
        // an infinity or NaN in a key's place is not 0)
        const int seen = r0 + 4 * ty + shift - k0;  // last key of the tile that the first of the four rows sees
        auto values = [&](auto masked) {
#pragma unroll 4
            for (int j = 0; j < BN; ++j) {
                const float4 pa = *reinterpret_cast<const float4 *>(ps + j * LD + 4 * ty);
                const float pr[4] = {pa.x, pa.y, pa.z, pa.w};
                ulonglong2 vb[C / 4];
#pragma unroll
                for (int c = 0; c < C / 4; ++c) vb[c] = *reinterpret_cast<const ulonglong2 *>(vs + j * D + 64 * c + 4 * tx);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (decltype(masked)::value && j > seen + i) continue;
                    const uint64_t pp = f2(pr[i], pr[i]);
#pragma unroll
                    for (int c = 0; c < C / 4; ++c) {
                        o[i][2 * c] = f2_fma(pp, vb[c].x, o[i][2 * c]);
                        o[i][2 * c + 1] = f2_fma(pp, vb[c].y, o[i][2 * c + 1]);
                    }
                }
            }
        };
        if (r0 + shift - k0 >= kn - 1)
            values(std::false_type{});
        else
            values(std::true_type{});
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float sum = l[i];
#pragma unroll
        for (int x = 8; x > 0; x >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, x);
        const int r = 4 * ty + i;
        if (r >= rows) continue;
        const float inv = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;  // no key: zeros; NaN stays
        const int64_t row = it.q_base + r0 + r;
        TO *out = reinterpret_cast<TO *>(a.out) + (row * a.Hq + h) * D;
#pragma unroll
        for (int c = 0; c < C / 4; ++c) {
            const float2 x = f2_get(o[i][2 * c]), y = f2_get(o[i][2 * c + 1]);
            store4(out + 64 * c + 4 * tx, make_float4(x.x * inv, x.y * inv, y.x * inv, y.y * inv));
        }
        if (tx == 0) {
            if (a.lse != nullptr) a.lse[h * a.q_total + row] = (m[i] + log2f(sum)) * kLn2;
            if (a.row_stat != nullptr) a.row_stat[h * a.q_total + row] = make_float2(m[i], inv);
        }
    }
}

// Threads are keys; rows of q in shared memory, kRows at a time.
constexpr int kWeightRows = 32;

template <int D>
__global__ void __launch_bounds__(kPackKeys) k_packed_weights(const PackedArgs a)
{
    __shared__ __align__(16) float qs[kWeightRows][D];
    __shared__ float2 st[kWeightRows];
    const PackItem it = a.key_items[blockIdx.x];
    const int g = blockIdx.y, j = it.row + threadIdx.x, shift = it.k_len - it.q_len;
    const bool there = j < it.k_len;
    float4 kr[D / 4];
    const float *k = reinterpret_cast<const float *>(a.k) + (int64_t)(it.k_base + (there ? j : it.row)) * a.k_stride + g * D;
#pragma unroll
    for (int d = 0; d < D / 4; ++d) kr[d] = load4(k + 4 * d);
    // rows that see the item's first key, of those that count
    const int first = max(max(0, it.q_len - a.weight_rows), it.row - shift);
    float w = 0.f;
    for (int h = g * a.G; h < (g + 1) * a.G; ++h) {
        for (int i0 = first; i0 < it.q_len; i0 += kWeightRows) {
            const int n = min(kWeightRows, it.q_len - i0);
            __syncthreads();
            for (int t = threadIdx.x; t < n * (D / 4); t += kPackKeys) {
                const int r = t / (D / 4), d = t % (D / 4) * 4;
                store4(&qs[r][d], load4(reinterpret_cast<const float *>(a.q) + (int64_t)(it.q_base + i0 + r) * a.q_stride + h * D + d));
            }
            if (threadIdx.x < n) st[threadIdx.x] = a.row_stat[(int64_t)h * a.q_total + it.q_base + i0 + threadIdx.x];
            __syncthreads();
            for (int r = 0; r < n; ++r) {
                float s[4] = {};
#pragma unroll
                for (int d = 0; d < D / 4; ++d) {
                    const float4 x = *reinterpret_cast<const float4 *>(&qs[r][4 * d]);
                    s[0] = fmaf(x.x, kr[d].x, s[0]);
                    s[1] = fmaf(x.y, kr[d].y, s[1]);
                    s[2] = fmaf(x.z, kr[d].z, s[2]);
                    s[3] = fmaf(x.w, kr[d].w, s[3]);
                }
                const float2 ml = st[r];
                if (there && j <= i0 + r + shift) w += exp2f(((s[0] + s[1]) + (s[2] + s[3])) * a.scale_log2 - ml.x) * ml.y;
            }
        }
    }
    if (there) a.key_weight[(int64_t)g * a.k_total + it.k_base + j] = w;
}

template <typename TO, int D>
cudaError_t launch(const PackedArgs &a, cudaStream_t s)
{
    auto kern = k_packed_f32<TO, D>;
    constexpr int bytes = (2 * D * LD + BN * D) * (int)sizeof(float);
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != cudaSuccess) return e;
    kern<<<(unsigned)((int64_t)a.n_items * kHalves * a.Hq), kThreads, bytes, s>>>(a);
    note_launch();
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_packed_f32(const PackedArgs &a, int D, int out_dtype, cudaStream_t s)
{
    if (out_dtype == RIS_F32) return D == 128 ? launch<float, 128>(a, s) : launch<float, 64>(a, s);
    return D == 128 ? launch<__nv_bfloat16, 128>(a, s) : launch<__nv_bfloat16, 64>(a, s);
}

cudaError_t launch_packed_weights_f32(const PackedArgs &a, int D, cudaStream_t s)
{
    const dim3 grid((unsigned)a.n_key_items, (unsigned)a.Hkv);
    if (D == 128)
        k_packed_weights<128><<<grid, kPackKeys, 0, s>>>(a);
    else
        k_packed_weights<64><<<grid, kPackKeys, 0, s>>>(a);
    note_launch();
    return cudaGetLastError();
}

}  // namespace ris
