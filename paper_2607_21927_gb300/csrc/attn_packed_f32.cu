// Causal attention over packed prompts on the FP32 pipe: fp32 inputs, which never pass through a
// narrower product, and the weight that each key got from a sequence's last rows.
//
// k_packed_f32: one CTA per (32 query rows, query head) walks the keys in tiles of 64 with a running
// maximum and sum. Keys and values come row by row by cp.async into a buffer each, so that the next keys
// travel under the value product and the next values under the scores; rows of 4 more elements than the
// head dim keep 16-byte reads of eight neighbouring rows apart. S: a 4 x 4 patch per thread, 4 elements of
// d at a time as packed pairs (which leaves two partial sums per score); the softmax over the 16 lanes that
// share a row; O += P V with a 4 x D/16 patch, P as pairs of the same weight in shared memory (two moves a
// weight otherwise). Bound by the FMA pipe: 4 D flops per pair and head; shared memory reads fill three
// quarters of its bandwidth beside it. 900 rows behind 301 keys at 12 / 2 heads of 128 take 133 us, 31 of
// 78 TFLOP/s: the pipe is 53 % busy while an SM has work (two warps to a scheduler, each a patch of 212
// registers), and a fifth of the time goes to the uneven ends. Tiles of 32 rows, because a short prompt has
// few of them and the one with the most keys is the last to end.
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

constexpr int BM = 32, BN = 64, LP = 2 * BN + 4;  // rows and keys of a tile, pitch of P
constexpr int kThreads = 4 * BM;
constexpr int kParts = kPackRows / BM;

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

// R rows of one head from memory to rows of pitch D + 4 (PAD) or D in shared memory, asynchronously; rows
// past `rows` as zeros
template <int R, int D, bool PAD>
__device__ __forceinline__ void fetch_rows(float *dst, const float *x, int64_t stride, int rows)
{
#pragma unroll
    for (int e = 0; e < R * (D / 4) / kThreads; ++e) {
        const int t = threadIdx.x + e * kThreads, r = t / (D / 4), d = t % (D / 4) * 4;
        const uint32_t to = (uint32_t)__cvta_generic_to_shared(dst + r * (PAD ? D + 4 : D) + d);
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(x + (r < rows ? r : 0) * stride + d), "r"(r < rows ? 16 : 0)
                     : "memory");
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
}
template <int N>
__device__ __forceinline__ void fetched_but()  // all but the last N groups
{
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

template <typename TO, int D>
__global__ void __launch_bounds__(kThreads, 2) k_packed_f32(const PackedArgs a)
{
    constexpr int LK = D + 4;
    extern __shared__ __align__(16) float sm[];
    float *const qs = sm, *const ks = qs + BM * LK, *const vs = ks + BN * LK, *const ps = vs + BN * D;
    // (what follows is not let in early: its CTAs, in the places of those that end first, would upset the
    // order by length of a next call's: 157 us instead of 135)
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int b = blockIdx.x, h = b % a.Hq, part = kParts - 1 - b / a.Hq % kParts;
    const PackItem it = a.items[b / a.Hq / kParts];
    const int r0 = it.row + part * BM, rows = min(BM, it.q_len - r0);
    if (rows <= 0) return;
    const int g = h / a.G;
    const int shift = it.k_len - it.q_len;              // row i sees keys j <= i + shift
    const int keys = max(0, min(it.k_len, r0 + rows + shift));  // that the last of the rows sees
    const float *q = reinterpret_cast<const float *>(a.q) + (int64_t)(it.q_base + r0) * a.q_stride + h * D;
    const float *k = reinterpret_cast<const float *>(a.k) + (int64_t)it.k_base * a.k_stride + g * D;
    const float *v = reinterpret_cast<const float *>(a.v) + (int64_t)it.k_base * a.v_stride + g * D;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;  // rows 4 ty + i; keys tx + 16 j; columns 4 tx + 64 c
    fetch_rows<BM, D, true>(qs, q, a.q_stride, rows);
    if (keys > 0) {
        fetch_rows<BN, D, true>(ks, k, a.k_stride, min(BN, keys));
        fetch_rows<BN, D, false>(vs, v, a.v_stride, min(BN, keys));
    }
    constexpr int C = D / 16;  // columns of O of a thread
    uint64_t o[4][C / 2] = {};
    float m[4], l[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) m[i] = -INFINITY, l[i] = 0.f;
    for (int k0 = 0; k0 < keys; k0 += BN) {
        const int kn = min(BN, keys - k0), left = min(BN, keys - k0 - BN);  // keys of this tile and of the next one
        fetched_but<1>();  // (the values' copy may still be on its way)
        __syncthreads();
        uint64_t s2[4][4] = {};  // two partial sums of each score: of the even and of the odd elements
#pragma unroll 4
        for (int d = 0; d < D; d += 4) {
            ulonglong2 qa[4], kb[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) qa[i] = *reinterpret_cast<const ulonglong2 *>(qs + (4 * ty + i) * LK + d);
#pragma unroll
            for (int j = 0; j < 4; ++j) kb[j] = *reinterpret_cast<const ulonglong2 *>(ks + (tx + 16 * j) * LK + d);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    s2[i][j] = f2_fma(qa[i].x, kb[j].x, s2[i][j]);
                    s2[i][j] = f2_fma(qa[i].y, kb[j].y, s2[i][j]);
                }
        }
        __syncthreads();  // the keys' buffer is free
        if (left > 0)
            fetch_rows<BN, D, true>(ks, k + (int64_t)(k0 + BN) * a.k_stride, a.k_stride, left);
        else
            asm volatile("cp.async.commit_group;" ::: "memory");
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int last = r0 + 4 * ty + i + shift - k0;  // last key of the tile that the row sees
            float s[4], mx = -INFINITY;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 x = f2_get(s2[i][j]);
                const int key = tx + 16 * j;
                s[j] = key <= last && key < kn ? (x.x + x.y) * a.scale_log2 : -INFINITY;
                mx = fmaxf(mx, s[j]);
            }
#pragma unroll
            for (int x = 8; x > 0; x >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, x));
            const float nm = fmaxf(m[i], mx), ref = nm == -INFINITY ? 0.f : nm;
            const float al = exp2f(m[i] - ref);
            m[i] = nm;
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[j] = exp2f(s[j] - ref);
                sum += s[j];
                *reinterpret_cast<uint64_t *>(ps + (4 * ty + i) * LP + 2 * (tx + 16 * j)) = f2(s[j], s[j]);
            }
            l[i] = fmaf(l[i], al, sum);  // this lane's part of the row's sum
            const uint64_t al2 = f2(al, al);
#pragma unroll
            for (int c = 0; c < C / 2; ++c) o[i][c] = f2_mul(o[i][c], al2);
        }
        fetched_but<1>();  // (the next keys' copy may still be on its way)
        __syncthreads();
        // O += P V; where some row does not see the whole tile, a row takes only the keys that it sees (0 times
        // an infinity or NaN in a key's place is not 0)
        const int seen = r0 + 4 * ty + shift - k0;  // last key of the tile that the first of the four rows sees
        auto values = [&](auto masked) {
#pragma unroll 4
            for (int j = 0; j < BN; j += 2) {
                ulonglong2 pa[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) pa[i] = *reinterpret_cast<const ulonglong2 *>(ps + (4 * ty + i) * LP + 2 * j);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    ulonglong2 vb[C / 4];
#pragma unroll
                    for (int c = 0; c < C / 4; ++c) vb[c] = *reinterpret_cast<const ulonglong2 *>(vs + (j + e) * D + 64 * c + 4 * tx);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (decltype(masked)::value && j + e > seen + i) continue;
                        const uint64_t pp = e == 0 ? pa[i].x : pa[i].y;
#pragma unroll
                        for (int c = 0; c < C / 4; ++c) {
                            o[i][2 * c] = f2_fma(pp, vb[c].x, o[i][2 * c]);
                            o[i][2 * c + 1] = f2_fma(pp, vb[c].y, o[i][2 * c + 1]);
                        }
                    }
                }
            }
        };
        if (r0 + shift - k0 >= kn - 1)
            values(std::false_type{});
        else
            values(std::true_type{});
        __syncthreads();  // the values' buffer and P's are free
        if (left > 0)
            fetch_rows<BN, D, false>(vs, v + (int64_t)(k0 + BN) * a.v_stride, a.v_stride, left);
        else
            asm volatile("cp.async.commit_group;" ::: "memory");
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
    after_last();
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
    constexpr int bytes = ((BM + BN) * (D + 4) + BN * D + BM * LP) * (int)sizeof(float);
    static Once once;
    const cudaError_t ready = once([&] { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes); });
    if (ready != cudaSuccess) return ready;
    return launch_chained(kern, dim3((unsigned)((int64_t)a.n_items * kParts * a.Hq)), dim3(kThreads), bytes, s, a);
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
    return launch_chained(D == 128 ? k_packed_weights<128> : k_packed_weights<64>, grid, dim3(kPackKeys), 0, s, a);
}

}  // namespace ris
