// Causal attention over packed prompts on the 5th-generation tensor cores, bf16 inputs.
//
// S = Q K^T with bf16 operands (exact products, fp32 sums), one online softmax per row over the keys j <= i
// + k_len - q_len of its own sequence, O = P V with P as fp16 (11 bits; a bf16 P would add as much error
// again as the bf16 output's own rounding) against the values as fp16 scaled by a power of two of their
// sequence and KV head (a bf16 value is exact there down to 2^-30 of the largest), the row's sum from the
// fp32 weights before they are rounded. The values are converted by two passes over V ahead of the
// attention (bounds, then the values): a few percent of a call where there are as many rows as keys, as V
// is read once per 128 rows of it anyway; most of one of few rows behind many keys.
//
// A work item is a tile of 128 rows of a sequence, the ones with the most keys first. Two kernels:
//   k_packed_rows  head dim 64, and short prompts at head dim 128: persistent, two CTAs to an SM, each
//                  with a row tile at a time
//   k_packed128    long prompts at head dim 128: two CTAs of a cluster share every key and value tile
//
// Every mbarrier wait is bounded; a wait that gives up sets the device error word, every role falls
// through to the end, TMEM is released and the CTA returns.
//
// Where a sequence's values of a KV head are not all finite (0 times an infinity is not 0, and a product
// over a tile multiplies keys that a row does not see by 0) or differ too much for fp16, its rows are
// computed from the inputs as given, on the FP32 pipe, each over exactly the keys it sees; and so are rows
// of scores too large for P's range.
#include <cuda.h>
#include <cudaTypedefs.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cstddef>
#include <cstdint>
#include <mutex>
#include <type_traits>

#include "attn_common.cuh"
#include "row_tiles.cuh"
#include "serve.h"

namespace ris {

// Device error word of this file (bit 1: a bounded wait gave up); read by ris_device_status.
__device__ unsigned int g_ris_packed_error;

namespace {

using namespace tc;

constexpr int BM = kTileRows, BN = kTileKeys;
static_assert(kPackRows == BM, "an item is a row tile");
constexpr int kGroupWarps = 4;     // of a softmax group: one thread per row
constexpr int kSoftmaxWarps = 2 * kGroupWarps;
constexpr int kTmaWarp = kSoftmaxWarps, kScoreWarp = kSoftmaxWarps + 1, kValueWarp = kSoftmaxWarps + 2,
              kRelayWarp = kSoftmaxWarps + 3;
constexpr int kThreads = 32 * (kSoftmaxWarps + 4);
// registers per thread: at launch, then after setmaxnreg of a softmax and of a loader / MMA thread
constexpr int kRegs = 168, kSoftmaxRegs = 200, kOtherRegs = 104;
static_assert(2 * kSoftmaxRegs + kOtherRegs == 3 * kRegs, "the shares of the three warpgroups add up to the launch's");
// The reference m of a row moves only when its maximum grows by more than kLazyLog2. P = 2^(s - m +
// kAboveLog2) stays below 2^15 and keeps fp16's 11 bits down to 2^-21 of the reference: rows whose weight
// goes to one key with next to no value are made of such.
constexpr float kLazyLog2 = 7.f, kAboveLog2 = 7.f;
// P's exponent is rounded once, the maximum behind m was rounded as a product: up to here they agree well
// enough for P's bound. Rows that pass it (no model's do) are computed on the FP32 pipe, where products are
// rounded alike.
constexpr float kFarLog2 = 0x1p23f;
constexpr uint32_t kTmemCols = 512;

// Exponent E of the values' scale 2^-E: the largest magnitude lands in [2^13, 2^14).
__device__ __forceinline__ int value_exp(float vmax)
{
    return min(max((int)((__float_as_uint(vmax) >> 23) & 0xFF) - 127 - 13, -100), 114);
}

// P = 2^(s sc - mu + kAboveLog2) of columns C0 .. C1 - 1 as fp16, two keys to a word, and the sum of the
// weights before they are rounded
template <int C0 = 0, int C1 = BN>
__device__ __forceinline__ float weights_of(const float (&sv)[BN], float sc, float mu, uint32_t (&hw)[BN / 2])
{
    const uint64_t sc2 = f2_pack(sc, sc), nmu2 = f2_pack(kAboveLog2 - mu, kAboveLog2 - mu);
    uint64_t sum[2] = {0, 0};
#pragma unroll
    for (int w = C0 / 2; w < C1 / 2; ++w) {
        float x0, x1;
        f2_unpack(f2_fma(f2_pack(sv[2 * w], sv[2 * w + 1]), sc2, nmu2), x0, x1);
        x0 = ex2(x0);
        x1 = ex2(x1);
        const __half2 hp = __floats2half2_rn(x0, x1);
        sum[w & 1] = f2_add(sum[w & 1], f2_pack(x0, x1));
        hw[w] = *reinterpret_cast<const uint32_t *>(&hp);
    }
    float a, b;
    f2_unpack(f2_add(sum[0], sum[1]), a, b);
    return a + b;
}

// A row's softmax as the other outputs: log-sum-exp, and (maximum, 1 / sum) for the key weights.
__device__ __forceinline__ float inverse_sum(float l) { return l > 0.f ? 1.f / l : l == 0.f ? 0.f : l; }
__device__ __forceinline__ void store_row(const PackedArgs &a, int h, int64_t row, float m, float l)
{
    if (a.lse != nullptr) a.lse[h * a.q_total + row] = (m + log2f(l)) * kLn2;
    if (a.row_stat != nullptr) a.row_stat[h * a.q_total + row] = make_float2(m, inverse_sum(l));
}
// The same of a row that is computed from the inputs as given: the key weights take their scores from
// tiles, so the maximum that goes with them is the tiles' own (`top`), and only the sum the row's.
__device__ __forceinline__ void store_top(const PackedArgs &a, int h, int64_t row, float top)
{
    if (a.row_stat != nullptr) a.row_stat[h * a.q_total + row].x = top;
}
__device__ __forceinline__ void store_given(const PackedArgs &a, int h, int64_t row, float m, float l)
{
    if (a.lse != nullptr) a.lse[h * a.q_total + row] = (m + log2f(l)) * kLn2;
    if (a.row_stat != nullptr) a.row_stat[h * a.q_total + row].y = inverse_sum(l);
}

// Rows on the FP32 pipe from the inputs as given: kGivenRows of them from i0 on, then those `step` later,
// up to row i1 of the item's sequence, by one warp over the keys that each sees (a lane per key for the
// scores, per channels for the outputs), through kGivenFloats of shared memory. With `stats` the other
// outputs too, else those of the tiles stand: a row's maximum and sum do not depend on the values. 8,192
// tokens of one prompt, one of two KV heads so: 8.3 ms (eight rows together 5.5, but the row tiles then
// took 1.5 % more for their registers; a row by itself 120).
constexpr int kGivenRows = 4;
template <int D>
constexpr int kGivenFloats = kGivenRows * D + 32 * kGivenRows;
template <int DT, typename TOut>
__device__ __noinline__ void rows_as_given(const PackedArgs &a, const PackItem &it, int i0, int i1, int step, int h, float *mem, bool stats)
{
    constexpr int R = kGivenRows, C = DT / 32;
    const int lane = threadIdx.x & 31, g = h / a.G, shift = it.k_len - it.q_len;
    const __nv_bfloat16 *k = reinterpret_cast<const __nv_bfloat16 *>(a.k) + (int64_t)it.k_base * a.k_stride + g * DT;
    const __nv_bfloat16 *v = reinterpret_cast<const __nv_bfloat16 *>(a.v) + (int64_t)it.k_base * a.v_stride + g * DT + C * lane;
    float *const qs = mem, *const ps = qs + R * DT;  // [row][channel], [key][row]
    auto value = [](uint32_t w, int e) { return __uint_as_float((e & 1) ? (w & 0xFFFF0000u) : (w << 16)); };
    i1 = min(i1, it.q_len);
    for (; i0 < i1; i0 += step) {
        const int rows = min(R, i1 - i0);
        __syncwarp();
        for (int t = lane; t < R * DT / 8; t += 32) {
            const int r = t / (DT / 8), d = t % (DT / 8) * 8;
            const __nv_bfloat16 *q = reinterpret_cast<const __nv_bfloat16 *>(a.q) + (int64_t)(it.q_base + i0 + min(r, rows - 1)) * a.q_stride + h * DT + d;
            const uint4 x = *reinterpret_cast<const uint4 *>(q);
            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int e = 0; e < 8; ++e) qs[r * DT + d + e] = value(w[e >> 1], e);
        }
        __syncwarp();
        float m[R], l[R], o[R][C];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            m[r] = -INFINITY, l[r] = 0.f;
#pragma unroll
            for (int c = 0; c < C; ++c) o[r][c] = 0.f;
        }
        const int n = min(it.k_len, i0 + rows + shift);  // keys that the last of the rows sees
        for (int j0 = 0; j0 < n; j0 += 32) {
            const int j = j0 + lane;
            const __nv_bfloat16 *kj = k + (int64_t)min(j, n - 1) * a.k_stride;
            float s[R] = {};
#pragma unroll 2
            for (int d = 0; d < DT; d += 8) {
                const uint4 x = *reinterpret_cast<const uint4 *>(kj + d);
                const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const float4 qa = *reinterpret_cast<const float4 *>(qs + r * DT + d), qb = *reinterpret_cast<const float4 *>(qs + r * DT + d + 4);
                    s[r] = fmaf(qa.x, value(w[0], 0), fmaf(qa.y, value(w[0], 1), fmaf(qa.z, value(w[1], 0), fmaf(qa.w, value(w[1], 1), s[r]))));
                    s[r] = fmaf(qb.x, value(w[2], 0), fmaf(qb.y, value(w[2], 1), fmaf(qb.z, value(w[3], 0), fmaf(qb.w, value(w[3], 1), s[r]))));
                }
            }
            float p[R];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float x = r < rows && j <= i0 + r + shift ? __fmul_rn(s[r], a.scale_log2) : -INFINITY;
                const float nm = fmaxf(m[r], warp_max(x)), ref = nm == -INFINITY ? 0.f : nm, al = exp2f(m[r] - ref);
                p[r] = exp2f(x - ref);
                m[r] = nm;
                l[r] = fmaf(l[r], al, p[r]);  // this lane's part of the row's sum
#pragma unroll
                for (int c = 0; c < C; ++c) o[r][c] *= al;
            }
#pragma unroll
            for (int r = 0; r < R; r += 4) *reinterpret_cast<float4 *>(ps + lane * R + r) = make_float4(p[r], p[r + 1], p[r + 2], p[r + 3]);
            __syncwarp();
            // (a row takes only the keys that it sees: 0 times an infinity or NaN in a key's place is not 0)
            auto add = [&](auto whole) {
#pragma unroll 4
                for (int e = 0; e < 32; ++e) {
                    if (!decltype(whole)::value && j0 + e >= n) break;
                    const __nv_bfloat16 *ve = v + (int64_t)(j0 + e) * a.v_stride;
                    uint32_t w[C / 2];
                    if constexpr (C == 4) {
                        const uint2 x = *reinterpret_cast<const uint2 *>(ve);
                        w[0] = x.x, w[1] = x.y;
                    } else {
                        w[0] = *reinterpret_cast<const uint32_t *>(ve);
                    }
                    float pe[R];
#pragma unroll
                    for (int r = 0; r < R; r += 4) {
                        const float4 x = *reinterpret_cast<const float4 *>(ps + e * R + r);
                        pe[r] = x.x, pe[r + 1] = x.y, pe[r + 2] = x.z, pe[r + 3] = x.w;
                    }
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        if (!decltype(whole)::value && (r >= rows || j0 + e > i0 + r + shift)) continue;
#pragma unroll
                        for (int c = 0; c < C; ++c) o[r][c] = fmaf(pe[r], value(w[c / 2], c), o[r][c]);
                    }
                }
            };
            if (rows == R && j0 + 31 <= i0 + shift)
                add(std::true_type{});
            else
                add(std::false_type{});
            __syncwarp();
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float sum = warp_sum(l[r]);
            if (r >= rows) continue;
            if (stats && lane == 0) store_given(a, h, it.q_base + i0 + r, m[r], sum);
            TOut *out = reinterpret_cast<TOut *>(a.out) + ((int64_t)(it.q_base + i0 + r) * a.Hq + h) * DT + C * lane;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const float x = sum == 0.f ? 0.f : o[r][c] / sum;
                if constexpr (sizeof(TOut) == 4)
                    out[c] = x;
                else
                    out[c] = __float2bfloat16_rn(x);
            }
        }
    }
}

struct PackedMaps {
    CUtensorMap q, k, v, out;
};

// The kernels that lay out the values (k_values_f16) have finished. Ahead of it run the start-up and, as
// nothing before this call is still running (see there), the copies of queries and keys and the first
// scores.
__device__ __forceinline__ void values_ready() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// O of 32 rows (a warp's) x OC columns from TMEM, normalised, into the warp's part of shared memory, row by
// row in 16-byte pieces swizzled by the row (128-byte rows: as TMA reads a box). Rows with no weight (inv
// 0) become zeros whatever the columns hold.
template <int OC, typename TOut>
__device__ __forceinline__ void stage_out(unsigned char *stage, uint32_t t_o, float inv)
{
    constexpr int RB = OC * (int)sizeof(TOut), NP = RB / 16;  // bytes and pieces of a row's part
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int c0 = 0; c0 < OC; c0 += 32) {
        float ov[32];
        tmem_ld32(t_o + c0, ov);
#pragma unroll
        for (int c = 0; c < 32; ++c) ov[c] = inv == 0.f ? 0.f : ov[c] * inv;
#pragma unroll
        for (int e = 0; e < 32 * (int)sizeof(TOut) / 16; ++e) {
            const int piece = c0 * (int)sizeof(TOut) / 16 + e;
            store16<TOut>(stage + lane * RB + ((piece ^ (lane & (NP - 1))) << 4), ov + e * (16 / (int)sizeof(TOut)));
        }
    }
}
// the first `rows` of those rows to memory, so that neighbouring lanes store neighbouring pieces of a row
template <int OC, typename TOut>
__device__ __forceinline__ void rows_out(const unsigned char *stage, TOut *out, int64_t pitch, int rows)
{
    constexpr int RB = OC * (int)sizeof(TOut), NP = RB / 16;
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int e = 0; e < NP; ++e) {
        const int rr = e * (32 / NP) + lane / NP, piece = lane & (NP - 1);
        const uint4 x = *reinterpret_cast<const uint4 *>(stage + rr * RB + ((piece ^ (rr & (NP - 1))) << 4));
        if (rr < rows) *reinterpret_cast<uint4 *>(out + rr * pitch + piece * (16 / (int)sizeof(TOut))) = x;
    }
    __syncwarp();
}

// What the warps of a cluster leave in each of its CTAs for the end of the kernel.
struct ClosingNotes {
    uint32_t bad;        // a wait gave up in either CTA
    uint32_t scored;     // tiles whose score products were issued and committed
    uint32_t valued;     // tiles whose value products were
    uint32_t keys[2], values[2];  // tiles whose keys / values each CTA requested (in the first CTA)
};

// ---------------------------------------------------------------- head dim 128
// Shared memory (bytes, from a 1024-aligned base).
struct Lay128 {
    static constexpr int DT = 128, NSK = 4, NSV = 4;  // stages of the key and of the value ring
    static constexpr int KROWS = BN / 2;           // keys of a tile held by one CTA
    static constexpr int K_BLK = KROWS * 128;      // one 64-column block
    static constexpr int K_STAGE = 2 * K_BLK;
    static constexpr int V_STAGE = BN * 128;       // 64 of the 128 value columns
    static constexpr int Q_BLK = BM * 128;
    static constexpr int OFF_K = 0;
    static constexpr int OFF_V = NSK * K_STAGE;
    static constexpr int OFF_Q = OFF_V + NSV * V_STAGE;
    static constexpr int OFF_BARS = OFF_Q + 2 * Q_BLK;
    static constexpr int OFF_TMEM = OFF_BARS + 224;  // after the barriers
    static constexpr int OFF_END = OFF_TMEM + 4;     // ClosingNotes
    static constexpr int OFF_M = OFF_BARS + 256;     // float [BM]
    static constexpr int OFF_ML = OFF_M + BM * 4;    // float2 [2][BM]
    static constexpr int OFF_TOP = OFF_ML + 2 * BM * 8;  // float [2][BM]
    static constexpr int BYTES = OFF_TOP + 2 * BM * 4;
    static_assert(BYTES <= 232448 && OFF_END + (int)sizeof(ClosingNotes) <= OFF_M, "shared memory of a CTA");
    // Barriers, one of each kind per ring stage or buffer, so that no waiter can fall two phases behind a
    // barrier it polls by parity:
    //   Q_FULL          the query tiles have landed (relayed with the first keys)
    //   K_FULL, V_FULL  a tile's keys / values have landed (relayed to S_GO / P_GO)
    //   S_GO            the score products of a tile may start: its keys have landed and the scores
    //                   of the tile two before (if any) have been read out of their buffer
    //   S_FULL          they are done (and the key stage is free)
    //   P_GO            the value product may start: P is written and the values have landed
    //   PV_DONE         it is done (P's buffer and the value stage are free, O has settled)
    // S_FULL and PV_DONE of each CTA get the products' completion. The others are used in the
    // cluster's first CTA, whose warps issue the products: the loaders of both CTAs announce
    // their copies there and the copies complete there, and the softmax warps of both arrive there.
    static constexpr int B_Q_FULL = 0, B_K_FULL = 1, B_S_GO = B_K_FULL + NSK, B_S_FULL = B_S_GO + NSK,
                         B_V_FULL = B_S_FULL + NSK, B_P_GO = B_V_FULL + NSV, B_PV_DONE = B_P_GO + NSV,
                         NBAR = B_PV_DONE + NSV;
    static_assert(NBAR * 8 <= 224 && NBAR <= 32, "barriers below the TMEM base word, a lane each");
};

// Two CTAs of a cluster share their key and value tiles (tcgen05 cta_group::2, one 256 x 128 product over
// both SMs, each holding half of the B operand: 64 of a tile's keys, 64 of the value columns): two heads of a
// KV group on the same 128 rows or, where a group has an odd number of heads, two consecutive row
// tiles of a head. That halves what an SM reads of shared memory per product, which one CTA alone
// would need all of (128 B a clock), and the L2 traffic of the tiles.
//
//   warp 8 (TMA)    loads the query tile, then streams 128-key tiles of the keys and of the values
//                   into two rings, each CTA its half;
//   warp 11 (relay) (first CTA) passes what has landed on to the barriers of the issuing warps;
//   warps 9, 10     (first CTA) issue tcgen05.mma: the score tile S into a double-buffered TMEM score
//                   tile, and O += P V (A = P in TMEM, double-buffered) into the TMEM output tile;
//   warps 0-7       two groups of four warps, one thread per row in each, on alternate key tiles:
//                   scores from TMEM, causal cut (only where a warp's rows end inside the tile),
//                   maximum, fp32 online softmax from the reference maximum that the other group hands
//                   over, O rescaled in TMEM only when the maximum grew by more than 2^7, P into TMEM.
// TMEM: S 2 x 128 columns, O 128, P 2 x 64: all 512.
//
// Bounded by the tensor pipe: a tile pair takes 16 products of 256 x 128 x 16, 1,024 cycles. One prompt of
// 32,768 tokens at 12 / 2 heads: 1.96 ms, 1.68 PFLOP/s (cuBLAS 1.89 in a burst and 1.70 under the power
// limit), the pipe 87 % busy from the first CTA to the last.
template <typename TOut>
__global__ void __launch_bounds__(kThreads, 1) k_packed128(const __grid_constant__ PackedArgs a, const __grid_constant__ PackedMaps maps)
{
    using L = Lay128;
    constexpr int NSK = L::NSK, NSV = L::NSV, DT = 128;
    extern __shared__ __align__(1024) unsigned char smem[];
    uint64_t *const bars = reinterpret_cast<uint64_t *>(smem + L::OFF_BARS);
    uint32_t &tmem_base_sh = *reinterpret_cast<uint32_t *>(smem + L::OFF_TMEM);
    float *const m_sh = reinterpret_cast<float *>(smem + L::OFF_M);
    float2(*const ml_sh)[BM] = reinterpret_cast<float2(*)[BM]>(smem + L::OFF_ML);
    float(*const top_sh)[BM] = reinterpret_cast<float(*)[BM]>(smem + L::OFF_TOP);
    volatile ClosingNotes *const notes = reinterpret_cast<ClosingNotes *>(smem + L::OFF_END);
    const uint32_t sbase = smem_u32(smem);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const unsigned int *const gave_up = &g_ris_packed_error;

    // ---- the cluster's item: with an even group 128 rows of two heads, else 256 rows of one (rank 1 the
    // second half, which may hold no rows)
    const int rank = (int)(blockIdx.x & 1);
    const bool head_pair = (a.G & 1) == 0;
    const unsigned n_h = (unsigned)(head_pair ? a.Hq / 2 : a.Hq), c = blockIdx.x / 2, r2 = c / n_h;
    const int h = head_pair ? 2 * (int)(c - r2 * n_h) + rank : (int)(c - r2 * n_h);
    const PackItem it = a.items[r2];
    const int q0 = it.row + (head_pair ? 0 : rank * BM);  // first row of this CTA, in its sequence
    const int g = h / a.G, shift = it.k_len - it.q_len;
    // keys that the last of the cluster's rows sees
    const int n_keys = max(0, min(it.k_len, min(it.q_len, it.row + (head_pair ? BM : 2 * BM)) + shift));
    const int n_kt = (n_keys + BN - 1) / BN;

    constexpr auto BAR = [](int i) { return (uint32_t)(L::OFF_BARS + 8 * i); };
    const bool first_loads = (sbase & 1023u) == 0u && n_kt > 0;
    if (warp == kTmaWarp) {
        if (lane < L::NBAR) {
            // S_GO, P_GO: the group's warps of each CTA and the relay; S_FULL, PV_DONE: the commit; the
            // copies' barriers: the loader of each CTA
            const bool go = (lane >= L::B_S_GO && lane < L::B_S_GO + NSK) || (lane >= L::B_P_GO && lane < L::B_P_GO + NSV);
            const bool done = (lane >= L::B_S_FULL && lane < L::B_S_FULL + NSK) || lane >= L::B_PV_DONE;
            mbar_init(smem_u32(&bars[lane]), go ? kGroupWarps * 2 + 1 : done ? 1 : 2);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        if (lane < (int)(sizeof(ClosingNotes) / 4)) reinterpret_cast<volatile uint32_t *>(smem + L::OFF_END)[lane] = 0u;
        __syncwarp();
        cluster_sync();  // the barriers of both CTAs are initialised once this is passed
        // the query tile and the first keys at once, under the rest of the start-up
        if (lane == 0 && first_loads) {
            const uint32_t lead = cluster_addr(sbase, 0);
            const uint32_t bq = lead + BAR(L::B_Q_FULL), bk = lead + BAR(L::B_K_FULL);
            const int key = it.k_base + L::KROWS * rank, row = it.q_base + q0;
            mbar_arrive_expect_tx<2>(bq, 2 * L::Q_BLK);
            mbar_arrive_expect_tx<2>(bk, L::K_STAGE);
            for (int blk = 0; blk < 2; ++blk) {
                tma_load_3d<2>(sbase + L::OFF_Q + blk * L::Q_BLK, &maps.q, 64 * blk, h, row, bq);
                tma_load_3d<2>(sbase + L::OFF_K + blk * L::K_BLK, &maps.k, 64 * blk, g, key, bk);
            }
        }
    } else {
        cluster_arrive();
        if (warp == kScoreWarp) tmem_alloc<2, kTmemCols>(smem_u32(&tmem_base_sh));  // by one full warp (of each CTA)
        cluster_wait();
    }
    const uint32_t lead = cluster_addr(sbase, 0);  // the issuing CTA's shared memory
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    // all 512 columns: the allocation starts at TMEM address 0, so every address below is a
    // constant (anything else ends the CTA as a failed wait does, below)
    constexpr uint32_t T_S0 = 0, T_O = T_S0 + 2 * BN, T_P0 = T_O + DT;
    static_assert(T_P0 + BN <= kTmemCols, "TMEM columns");
    const uint32_t tmem = tmem_base_sh;
    auto arrive_lead = [&](int bar) { mbar_arrive_cluster(lead + BAR(bar)); };
    bool ok = tmem == 0u && (sbase & 1023u) == 0u;  // (the swizzled boxes need the alignment)

    if (warp >= kSoftmaxWarps) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
    if (warp == kTmaWarp) {
        // =============================== TMA producer
        values_ready();
        if (lane == 0 && first_loads) {
            // (The query tile and the first keys were requested above.) Keys of tile j once the score
            // products of tile j - NSK are done, values of tile j once the value product of tile j - NSV
            // is: the loader waits on the barriers that announce those products (S_FULL, PV_DONE). The
            // score products of tile t + 1 finish before the value product of tile t, so in this order no
            // wait holds up a load that could go before it.
            int nk = 1, nv = 0;  // tiles whose keys / values were requested
            auto load_k = [&](int j) -> bool {
                if (j >= n_kt) return true;
                const int st = j % NSK;
                if (j >= NSK && !mbar_wait<2>(sbase + BAR(L::B_S_FULL + st), (j / NSK - 1) & 1, gave_up)) return false;
                const uint32_t bk = lead + BAR(L::B_K_FULL + st);
                const uint32_t dk = sbase + L::OFF_K + st * L::K_STAGE;
                mbar_arrive_expect_tx<2>(bk, L::K_STAGE);
                for (int blk = 0; blk < 2; ++blk)
                    tma_load_3d<2>(dk + blk * L::K_BLK, &maps.k, 64 * blk, g, it.k_base + j * BN + L::KROWS * rank, bk);
                nk = j + 1;
                return true;
            };
            auto load_v = [&](int j) -> bool {
                if (j >= n_kt) return true;
                const int st = j % NSV;
                if (j >= NSV && !mbar_wait<2>(sbase + BAR(L::B_PV_DONE + st), (j / NSV - 1) & 1, gave_up)) return false;
                const uint32_t bv = lead + BAR(L::B_V_FULL + st);
                mbar_arrive_expect_tx<2>(bv, L::V_STAGE);
                tma_load_3d<2>(sbase + L::OFF_V + st * L::V_STAGE, &maps.v, 64 * rank, g, it.k_base + j * BN, bv);
                nv = j + 1;
                return true;
            };
            ok = ok && load_v(0) && load_k(1) && load_v(1) && load_k(2) && load_v(2) && load_k(3) && load_v(3) && load_k(4);
            for (int t = 0; t < n_kt && ok; ++t) ok = load_k(t + 5) && load_v(t + 4);
            // (that the copies requested last have landed before a CTA leaves: see the end)
            st_cluster(sbase + L::OFF_END + offsetof(ClosingNotes, keys) + 4 * rank, 0, (uint32_t)nk);
            st_cluster(sbase + L::OFF_END + offsetof(ClosingNotes, values) + 4 * rank, 0, (uint32_t)nv);
            static_assert(NSK == 4 && NSV == 4, "the order of the loads and of the relay");
        }
    } else if (!ok || rank != 0) {
        // an unexpected base: straight to the common end; and the second CTA has nothing to issue
    } else if (warp == kRelayWarp) {
        // =============================== relay: what has landed, to the barriers that the issuing
        // warps wait on, in the order of the loads; so each of them waits on one barrier per tile
        if (lane == 0 && n_kt > 0) {
            auto relay_k = [&](int j) -> bool {
                if (j >= n_kt) return true;
                if (!mbar_wait<2>(sbase + BAR(L::B_K_FULL + j % NSK), (j / NSK) & 1, gave_up)) return false;
                mbar_arrive(sbase + BAR(L::B_S_GO + j % NSK));
                return true;
            };
            auto relay_v = [&](int j) -> bool {
                if (j >= n_kt) return true;
                if (!mbar_wait<2>(sbase + BAR(L::B_V_FULL + j % NSV), (j / NSV) & 1, gave_up)) return false;
                mbar_arrive(sbase + BAR(L::B_P_GO + j % NSV));
                return true;
            };
            ok = mbar_wait<2>(sbase + BAR(L::B_Q_FULL), 0, gave_up) && relay_k(0) && relay_v(0) && relay_k(1) && relay_v(1) &&
                 relay_k(2) && relay_v(2) && relay_k(3) && relay_v(3) && relay_k(4);
            for (int t = 0; t < n_kt && ok; ++t) ok = relay_k(t + 5) && relay_v(t + 4);
        }
    } else {
        // =============================== product issuers (of the cluster's first CTA, for both): one
        // warp for the scores, one for the value products. The whole warp runs this code, so that every operand
        // is warp-uniform, and one elected lane issues.
        constexpr uint32_t ID_S = idesc_bf16(2 * BM, BN, false);  // S[128 x 128] = Q K^T, both K-major
        constexpr uint32_t ID_O = idesc_f16(2 * BM, DT, true);    // O[128 x 128] += P V, fp16, V MN-major
        // score products of a tile of ring stage ST: a k-step of 16 columns 32 B further in a 128 B row
        auto issue_s = [&](auto st_c) {
            constexpr int ST = decltype(st_c)::value;
            const uint32_t kd = desc_lo(sbase + L::OFF_K + ST * L::K_STAGE, 16);
            const uint32_t qd = desc_lo(sbase + L::OFF_Q, 16);
            constexpr uint32_t dt = T_S0 + (ST & 1) * BN;
            if (elect_one()) {
#pragma unroll
                for (int ks = 0; ks < DT / 16; ++ks)
                    tc_mma_ss<2>(dt, qd + dstep((ks >> 2) * L::Q_BLK + (ks & 3) * 32), kd + dstep((ks >> 2) * L::K_BLK + (ks & 3) * 32), ID_S,
                                 ks > 0);
                tc_commit<2>(sbase + BAR(L::B_S_FULL + ST));
            }
            __syncwarp();
        };
        // value product of a tile of ring stage ST: P (in TMEM, the buffer of the tile's parity), 128
        // keys packed two per column, times V, 128 keys x 128 B rows: 16 keys = two 8-row atoms (SBO 1024)
        auto issue_o = [&](auto st_c, uint32_t acc) {
            constexpr int ST = decltype(st_c)::value;
            const uint32_t vd = desc_lo(sbase + L::OFF_V + ST * L::V_STAGE, L::V_STAGE);
            if (elect_one()) {
#pragma unroll
                for (int ks = 0; ks < BN / 16; ++ks)
                    tc_mma_ts<2>(T_O, T_P0 + (ST & 1) * (BN / 2) + 8 * ks, vd + dstep(ks * 2048), ID_O, ks > 0 ? 1u : acc);
                tc_commit<2>(sbase + BAR(L::B_PV_DONE + ST));
            }
            __syncwarp();
        };
        auto wait_all = [&](int bar, int parity) -> bool {
            const bool got = __all_sync(0xFFFFFFFFu, mbar_wait<2>(sbase + BAR(bar), parity, gave_up));
            tc_fence_after();
            return got;
        };
        int issued = 0;  // tiles whose products this warp committed
        auto score_step = [&](auto st_c, int j) {
            if (!ok || j >= n_kt) return;
            ok = wait_all(L::B_S_GO + decltype(st_c)::value, (j / NSK) & 1);
            if (!ok) return;
            issue_s(st_c);
            issued = j + 1;
        };
        auto value_step = [&](auto st_c, int j) {
            if (!ok || j >= n_kt) return;
            ok = wait_all(L::B_P_GO + decltype(st_c)::value, (j / NSV) & 1);
            if (!ok) return;
            issue_o(st_c, j > 0 ? 1u : 0u);
            issued = j + 1;
        };
        using I0 = std::integral_constant<int, 0>;
        using I1 = std::integral_constant<int, 1>;
        using I2 = std::integral_constant<int, 2>;
        using I3 = std::integral_constant<int, 3>;
        if (warp == kScoreWarp) {
            for (int j = 0; j < n_kt && ok; j += 4) {
                score_step(I0{}, j);
                score_step(I1{}, j + 1);
                score_step(I2{}, j + 2);
                score_step(I3{}, j + 3);
            }
        } else {
            for (int j = 0; j < n_kt && ok; j += 4) {
                value_step(I0{}, j);
                value_step(I1{}, j + 1);
                value_step(I2{}, j + 2);
                value_step(I3{}, j + 3);
            }
        }
        if (lane < 2) {
            const int off = L::OFF_END + (warp == kValueWarp ? offsetof(ClosingNotes, valued) : offsetof(ClosingNotes, scored));
            st_cluster(sbase + off, lane, (uint32_t)issued);
        }
    }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
        // =============================== softmax: group grp of four warps takes the tiles of parity
        // grp, one thread per row q0 + r; at the end a thread owns half of its row's columns
        constexpr int OC = DT / 2;
        const int wq = warp & 3, grp = warp >> 2;
        const int r = wq * 32 + lane;  // TMEM lane
        const uint32_t lane_off = (uint32_t)(wq * 32) << 16;
        values_ready();
        const float sc = a.scale_log2, v_top = it.k_len > 0 ? a.v_top[(int64_t)it.seq * a.Hkv + g] : 0.f;
        // the group's score buffer is free for its first tile
        if (lane == 0 && grp < n_kt) arrive_lead(L::B_S_GO + grp);
        const int last_key = q0 + r + shift;          // last key that the row sees
        const int warp_sees = q0 + wq * 32 + shift;   // that every row of the warp sees (and those past the sequence's end)
        float l = 0.f, m_own = -INFINITY;  // row sum over this thread's tiles, relative to 2^m_own
        float far = 0.f, top = -INFINITY;  // largest magnitude of m; largest score
        bool s_full = false;  // seen at the end of the last tile: a poll takes 200 cycles even if it succeeds
        for (int j = grp; j < n_kt; j += 2) {
            if (ok) {
                const uint32_t bar = sbase + BAR(L::B_S_FULL + j % NSK);
                ok = __all_sync(0xFFFFFFFFu, s_full || mbar_wait<2, true>(bar, (j / NSK) & 1, gave_up));
            }
            tc_fence_after();
            uint32_t su[2][64];
            tmem_issue64(T_S0 + grp * BN + lane_off, su[0]);
            tmem_issue64(T_S0 + grp * BN + lane_off + 64, su[1]);
            tmem_wait_ld();
            pin64(su[0]);
            pin64(su[1]);
            tc_fence_before();
            __syncwarp();
            tc_fence_before();
            if (lane == 0 && j + 2 < n_kt) arrive_lead(L::B_S_GO + (j + 2) % NSK);
            float sv[BN];
#pragma unroll
            for (int e = 0; e < BN; ++e) sv[e] = __uint_as_float(su[e >> 6][e & 63]);
            if (warp_sees < j * BN + BN - 1) {
                uint32_t cw[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) cw[e] = causal_word(last_key - j * BN, e);
#pragma unroll
                for (int e = 0; e < BN; ++e) drop_unless(sv[e], cw[e >> 5], 1u << (e & 31));
            }
            const float mx = __fmul_rn(row_max(sv), sc);  // (the scale is positive)
            // The row's reference maximum moves on from tile to tile, handed to the other group. It moves, and
            // O is rescaled, only when the row max grows by more than kLazyLog2. The TMEM loads / stores are
            // warp-collective, so the whole warp runs them when any of its rows needs it.
            float m_prev = -INFINITY;
            if (j > 0) {
                pair_sync(1 + 2 * wq + (grp ^ 1));
                m_prev = m_sh[r];
            }
            const bool upd = mx > m_prev + kLazyLog2;
            const float m_ref = upd ? mx : m_prev, mu = m_ref == -INFINITY ? 0.f : m_ref;
            // the value product of tile t is done (t < 0: nothing to wait for)
            auto pv_done = [&](int t) -> bool {
                const uint32_t bar = sbase + BAR(L::B_PV_DONE + t % NSV);
                return t < 0 || __all_sync(0xFFFFFFFFu, mbar_wait<2, true>(bar, (t / NSV) & 1, gave_up));
            };
            const bool scale_o = upd && m_prev != -INFINITY;
            const bool any_scale = __any_sync(0xFFFFFFFFu, scale_o);
            const float al = scale_o ? exp2f(m_prev - m_ref) : 1.f;
            far = fmaxf(far, fabsf(mu));
            top = fmaxf(top, mx);
            if (m_ref != m_own) {
                l *= m_own == -INFINITY ? 0.f : exp2f(m_own - m_ref);
                m_own = m_ref;
            }
            uint32_t hw[BN / 2];
            const float lsum = weights_of(sv, sc, mu, hw);
            // Only now on to the other group: its exponentials (the other warp of this scheduler) run
            // while this warp stores P and takes the next tile's scores and maximum, and not
            // against this warp's own
            if (j + 1 < n_kt) {
                m_sh[r] = m_ref;
                __threadfence_block();
                pair_arrive(1 + 2 * wq + grp);
            }
            if (!ok) continue;
            ok = pv_done(j - 2);  // P's buffer is free
            if (!ok) continue;
            tc_fence_after();
            if (any_scale) {
                // O has settled once the value product of tile j - 1 is done (that of tile j - 2 first,
                // above, so that the barrier is not polled a phase early); nothing adds to it before
                // this warp's P is announced below, and the other group's warp of these rows scales it next
                // only after that product.
                ok = pv_done(j - 1);
                if (!ok) continue;
                tc_fence_after();
#pragma unroll 1
                for (int c0 = 0; c0 < DT; c0 += 32) {
                    float ov[32];
                    uint32_t ow[32];
                    tmem_ld32(T_O + lane_off + c0, ov);
#pragma unroll
                    for (int e = 0; e < 32; ++e) ow[e] = __float_as_uint(ov[e] * al);
                    tmem_st32(T_O + lane_off + c0, ow);
                }
                tmem_wait_st();
            }
            const uint32_t tp = T_P0 + grp * (BN / 2) + lane_off;
            tmem_st32(tp, hw);
            tmem_st32(tp + 32, hw + 32);
            s_full = j + 2 < n_kt && mbar_test<2, true>(sbase + BAR(L::B_S_FULL + (j + 2) % NSK), ((j + 2) / NSK) & 1);
            l += lsum;
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            tc_fence_before();
            if (lane == 0) arrive_lead(L::B_P_GO + j % NSV);
        }
        // the row's maximum and sum from both threads
        top_sh[grp][r] = top;
        ml_sh[grp][r] = make_float2(m_own, far > kFarLog2 && far < INFINITY ? INFINITY : l);  // (no sum of weights is infinite)
        ok = !pair_or(9 + wq, !ok);
        for (int t = max(0, n_kt - 2); t < n_kt && ok; ++t)  // in order, as above
            ok = __all_sync(0xFFFFFFFFu, mbar_wait<2>(sbase + BAR(L::B_PV_DONE + t % NSV), (t / NSV) & 1, gave_up));
        if (ok) {
            tc_fence_after();
            const float2 ma = ml_sh[0][r], mb = ml_sh[1][r];
            // the group of the last tile holds the final maximum; a group without tiles has l = 0
            const float m_fin = n_kt == 0 ? -INFINITY : ((n_kt - 1) & 1) ? mb.x : ma.x;
            const float lt = (ma.x == m_fin ? ma.y : ma.y * exp2f(ma.x - m_fin)) +
                             (mb.x == m_fin ? mb.y : mb.y * exp2f(mb.x - m_fin));
            const bool too_far = __any_sync(0xFFFFFFFFu, ma.y == INFINITY || mb.y == INFINITY);
            if (grp == 0 && q0 + r < it.q_len) {
                if (too_far)
                    store_top(a, h, it.q_base + q0 + r, fmaxf(top_sh[0][r], top_sh[1][r]));
                else
                    store_row(a, h, it.q_base + q0 + r, m_fin - kAboveLog2, lt);
            }
            // fp16 values were scaled by 2^-E for the value product
            if (v_top < INFINITY && !too_far) {
                const float inv = lt == 0.f ? 0.f : pow2i(value_exp(v_top)) / lt;
                const int w0 = q0 + 32 * wq;  // the warp's first row
                TOut *out = reinterpret_cast<TOut *>(a.out) + ((int64_t)(it.q_base + w0) * a.Hq + h) * DT + OC * grp;
                unsigned char *stage = smem + warp * (32 * OC * (int)sizeof(TOut));
                stage_out<OC, TOut>(stage, T_O + lane_off + OC * grp, inv);
                __syncwarp();
                rows_out<OC, TOut>(stage, out, (int64_t)a.Hq * DT, it.q_len - w0);
            } else {
                // (through the rings, as the outputs' way above)
                static_assert(kSoftmaxWarps * kGivenFloats<DT> * 4 <= L::OFF_Q, "the rings hold every warp's part");
                // (the pair of warps takes its own 32 rows)
                rows_as_given<DT, TOut>(a, it, q0 + 32 * wq + kGivenRows * grp, q0 + 32 * wq + 32, 2 * kGivenRows, h,
                                        reinterpret_cast<float *>(smem) + warp * kGivenFloats<DT>, too_far);
            }
        }
    }

    if (!ok) {
        atomicOr(&g_ris_packed_error, 2u);
        for (int x = 0; x < 2; ++x) st_cluster(sbase + L::OFF_END + offsetof(ClosingNotes, bad), x, 1u);
    }
    __syncwarp();
    tc_fence_before();
    // Neither CTA of a cluster may leave, or release TMEM, while a product is running or anything can
    // still reach its shared memory. The softmax warps of each CTA have seen, in their own
    // barriers, every commit (S_FULL of every tile, PV_DONE of every tile), and so the end of every copy:
    // nothing is under way unless a wait gave up. Then the copies and commits still to come, as the
    // loaders and the issuing warps counted them, are waited for before both CTAs leave. (What one
    // loader requested and the other did not is announced here in its place.)
    cluster_sync();
    __syncthreads();
    tc_fence_after();
    if (notes->bad != 0u) {
        if (warp == kTmaWarp && lane == 0) {
            auto landed = [&](int bar, int stages, int n0, int n1) {
                const int n = max(n0, n1);
                for (int j = max(0, n - stages); j < n; ++j) {
                    if (j >= min(n0, n1)) mbar_arrive(sbase + BAR(bar + j % stages));
                    mbar_wait_own<2>(sbase + BAR(bar + j % stages), (j / stages) & 1);
                }
            };
            if (rank == 0) {
                if (notes->keys[0] > 0u) mbar_wait_own<2>(sbase + BAR(L::B_Q_FULL), 0);
                landed(L::B_K_FULL, NSK, (int)notes->keys[0], (int)notes->keys[1]);
                landed(L::B_V_FULL, NSV, (int)notes->values[0], (int)notes->values[1]);
            }
            const int ns = (int)notes->scored, nv = (int)notes->valued;
            for (int j = max(0, ns - NSK); j < ns; ++j) mbar_wait_own<2>(sbase + BAR(L::B_S_FULL + j % NSK), (j / NSK) & 1);
            for (int j = max(0, nv - NSV); j < nv; ++j) mbar_wait_own<2>(sbase + BAR(L::B_PV_DONE + j % NSV), (j / NSV) & 1);
        }
        __syncwarp();
        cluster_sync();
        __syncthreads();
        tc_fence_after();
    }
    if (warp == kScoreWarp) tmem_dealloc<2, kTmemCols>(tmem);
}

// ---------------------------------------------------------------- a row tile per CTA at a time
template <int D>
struct LayRows {
    static constexpr int DT = D, NB = D / 64;              // 64-column blocks
    static constexpr bool OVER = D == 128;                 // P takes the scores' columns
    static constexpr int NSK = D == 64 ? 3 : 1, NSV = D == 64 ? 2 : 1, NI = 4;
    static constexpr int BLK = 128 * 128, TILE = NB * BLK; // 128 rows or keys of D 16-bit values
    static constexpr int OFF_K = 0, OFF_V = OFF_K + NSK * TILE, OFF_Q = OFF_V + NSV * TILE, OFF_OUT = OFF_Q + TILE,
                         OFF_BARS = OFF_OUT + BLK, OFF_INFO = OFF_BARS + 192, OFF_TMEM = OFF_INFO + NI * 64, BYTES = OFF_TMEM + 16;
    // Barriers, of a ring stage:
    //   K_FULL, V_FULL, Q_FULL  its keys / values / the query tile have landed
    //   K_FREE, V_FREE, Q_FREE  the products that read it are done
    //   I_FULL, I_FREE          a unit's description is there / every role has read it
    // and one phase per key tile:
    //   S_GO    the last scores have been read out of their buffer (only where P has its own columns:
    //           else the value product before has to be done, which says that too)
    //   S_FULL  the next are there
    //   P_GO    P is written (and O rescaled where needed)
    //   PV_DONE O has settled, P's buffer is free
    static constexpr int B_K_FULL = 0, B_V_FULL = B_K_FULL + NSK, B_Q_FULL = B_V_FULL + NSV, B_K_FREE = B_Q_FULL + 1,
                         B_V_FREE = B_K_FREE + NSK, B_Q_FREE = B_V_FREE + NSV, B_I_FULL = B_Q_FREE + 1, B_I_FREE = B_I_FULL + NI,
                         B_S_GO = B_I_FREE + NI, B_S_FULL = B_S_GO + 1, B_P_GO = B_S_FULL + 1, B_PV_DONE = B_P_GO + 1,
                         NBAR = B_PV_DONE + 1;
    static_assert(NBAR <= 24 && 2 * (BYTES + 1024) <= 228 * 1024, "barriers; two CTAs of an SM");
    static constexpr uint32_t COLS = 256, T_P = OVER ? 0 : BN, T_O = OVER ? BN : BN + BN / 2;  // TMEM; S at 0
    static_assert(T_O + DT <= COLS, "TMEM columns");
    // registers per thread: at launch, then after setmaxnreg of a softmax and of another thread
    static constexpr int THREADS = 256, REGS = 128, SOFTMAX_REGS = 200, OTHER_REGS = 56;
    static_assert(SOFTMAX_REGS + OTHER_REGS == 2 * REGS, "the shares of the two warpgroups add up to the launch's");
};

// What the other roles need to know of a unit, a (work item, query head).
struct UnitInfo {
    int n;                  // key tiles, -1: no more units
    int h, row, shift;      // head; first row; key j is seen by row i when j <= i + shift
    int q_base, q_len, k_base, k_len;
    int64_t id, top;        // its number; its place in v_top
};
static_assert(sizeof(UnitInfo) <= 64, "the ring's slots");

// The units of one CTA after another, in the items' order; the CTAs take them in rounds, every second round
// backwards, so that the long ones are dealt out evenly.
struct Units {
    int64_t total;
    int round;
    __device__ __forceinline__ bool next(const PackedArgs &a, PackItem &it, int &h, int64_t &id)
    {
        for (;;) {
            const int64_t base = (int64_t)++round * gridDim.x;
            if (base >= total) return false;
            const int64_t u = base + ((round & 1) ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
            if (u >= total) continue;
            it = a.items[(int)u / a.Hq];
            h = (int)u % a.Hq;
            id = u;
            return true;
        }
    }
};

// The rows of this CTA's units that are to be computed from the inputs as given: all of a unit's where the
// values ask for it, a warp's own 32 where their scores did (a.far).
template <int D, typename TOut>
__device__ __noinline__ void units_as_given(const PackedArgs &a, int warp, float *mem)
{
    Units units{(int64_t)a.n_items * a.Hq, -1};
    PackItem it;
    int h;
    int64_t id;
    while (units.next(a, it, h, id)) {
        if (it.k_len <= 0) continue;
        const bool far = a.far[id * kGroupWarps + warp] != 0;
        if (far) rows_as_given<D, TOut>(a, it, it.row + 32 * warp, it.row + 32 * warp + 32, kGivenRows, h, mem, true);
        if (!(a.v_top[(int64_t)it.seq * a.Hkv + h / a.G] < INFINITY))
            rows_as_given<D, TOut>(a, it, it.row + kGivenRows * warp, it.row + BM, kGivenRows * kGroupWarps, h, mem, false);
    }
}

// Persistent, two CTAs to an SM, each with one row tile at a time and one softmax group (TMEM 256 columns).
// A row tile of few keys is a chain of waits (copies, scores, softmax, value product, outputs: 5 us), and
// the two CTAs fill each other's; the loaders and issuing warps run on into the next unit while the last
// one is finished; the outputs leave by TMA. 64 prompts of 256 tokens take 40 us at 12 heads of 128, 58 at
// 32 heads of 64; with a CTA (head dim 128: a cluster) per unit they took 96 and 111. At head dim 64 a key
// tile's products and its 16,384 exponentials each take 512 cycles; it takes 1,050 an SM over 16,384 tokens
// (issue slots 57 %, exponentials 49 %, tensor pipe 49 % busy; 9 prompts of 16,233 tokens at 32 / 4 heads
// 188 us). It is the softmax warps' own chain at two warps to a scheduler, 2,110 cycles a tile: 1,000 for
// the weights (512 of exponentials, the other warp's in between), 390 for the maximum, 310 for the tensor
// memory's loads and stores with their fences, 350 from the loop's end to the next scores; half the
// products' work would take 1 % less time, no exponentials 18 %. Sixteen softmax warps to an SM instead of
// eight took 1,170, no maximum ahead of the weights 1,090. At head dim 128 the products of a CTA read as
// much shared memory as there is bandwidth, and long prompts go to k_packed128.
//
//   warp 4  the units, query and key tiles, warp 5 value tiles (TMA);
//   warp 6  S = Q K^T as soon as its columns are free, warp 7 O += P V;
//   warps 0-3  the softmax, one thread per row.
template <int D, typename TOut>
__global__ void __launch_bounds__(LayRows<D>::THREADS, 2) k_packed_rows(const __grid_constant__ PackedArgs a, const __grid_constant__ PackedMaps maps)
{
    using L = LayRows<D>;
    constexpr int NSK = L::NSK, NSV = L::NSV, NI = L::NI, NB = L::NB, TILE = L::TILE;
    constexpr int kLoadQK = 4, kLoadV = 5, kScores = 6, kValues = 7;
    extern __shared__ __align__(1024) unsigned char smem[];
    uint32_t &tmem_base_sh = *reinterpret_cast<uint32_t *>(smem + L::OFF_TMEM);
    const uint32_t sbase = smem_u32(smem);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const unsigned int *const gave_up = &g_ris_packed_error;
    auto bar = [&](int i) { return sbase + (uint32_t)(L::OFF_BARS + 8 * i); };
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    if (warp == kLoadQK) {
        if (lane < L::NBAR) {
            const bool by_group = lane == L::B_S_GO || lane == L::B_P_GO, free = lane >= L::B_I_FREE && lane < L::B_I_FREE + NI;
            mbar_init(bar(lane), by_group ? kGroupWarps : free ? kGroupWarps + 3 : 1);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
    } else if (warp == kScores) {
        tmem_alloc<1, L::COLS>(smem_u32(&tmem_base_sh));
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_base_sh;
    bool ok = (sbase & 1023u) == 0u;
    auto wait_all = [&](int i, int parity) -> bool {
        const bool got = __all_sync(0xFFFFFFFFu, mbar_wait<1>(bar(i), parity, gave_up));
        tc_fence_after();
        return got;
    };
    // description of unit u (a whole warp, or a loader's lane); its place is given back once every lane has it
    auto unit = [&](int u, UnitInfo &x) -> bool {
        if (!mbar_wait<1>(bar(L::B_I_FULL + u % NI), (u / NI) & 1, gave_up)) return false;
        x = *reinterpret_cast<const UnitInfo *>(smem + L::OFF_INFO + u % NI * 64);
        return true;
    };
    auto unit_read = [&](int u, bool one) { mbar_arrive_if(one, bar(L::B_I_FREE + u % NI)); };

    if (warp >= kGroupWarps) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(L::OTHER_REGS));
        if (warp == kLoadQK) {
            if (lane == 0 && ok) {
                Units units{(int64_t)a.n_items * a.Hq, -1};
                int nq = 0, nk = 0;  // query and key tiles asked for
                bool more = true;
                for (int u = 0; more && ok; ++u) {
                    PackItem it;
                    int h = 0, n = -1;
                    int64_t id = 0;
                    more = units.next(a, it, h, id);
                    if (u >= NI) ok = mbar_wait<1>(bar(L::B_I_FREE + u % NI), (u / NI - 1) & 1, gave_up);
                    if (!ok) break;
                    UnitInfo &x = *reinterpret_cast<UnitInfo *>(smem + L::OFF_INFO + u % NI * 64);
                    if (more) {
                        const int shift = it.k_len - it.q_len;
                        n = (max(0, min(it.k_len, min(it.q_len, it.row + BM) + shift)) + BN - 1) / BN;  // tiles that the rows see
                        x = UnitInfo{n, h, it.row, shift, it.q_base, it.q_len, it.k_base, it.k_len, id, (int64_t)it.seq * a.Hkv + h / a.G};
                    } else {
                        x.n = -1;
                    }
                    mbar_arrive(bar(L::B_I_FULL + u % NI));
                    const int g = h / a.G;
                    for (int j = 0; j < n; ++j, ++nk) {
                        const int st = nk % NSK;
                        if (nk >= NSK) ok = mbar_wait<1>(bar(L::B_K_FREE + st), (nk / NSK - 1) & 1, gave_up);
                        if (!ok) break;
                        mbar_arrive_expect_tx<1>(bar(L::B_K_FULL + st), TILE);
                        for (int blk = 0; blk < NB; ++blk)
                            tma_load_3d<1>(sbase + L::OFF_K + st * TILE + blk * L::BLK, &maps.k, 64 * blk, g, it.k_base + j * BN,
                                           bar(L::B_K_FULL + st));
                        if (j > 0) continue;
                        if (nq > 0) ok = mbar_wait<1>(bar(L::B_Q_FREE), (nq - 1) & 1, gave_up);
                        if (!ok) break;
                        mbar_arrive_expect_tx<1>(bar(L::B_Q_FULL), TILE);
                        for (int blk = 0; blk < NB; ++blk)
                            tma_load_3d<1>(sbase + L::OFF_Q + blk * L::BLK, &maps.q, 64 * blk, h, it.q_base + it.row, bar(L::B_Q_FULL));
                        ++nq;
                    }
                }
                // nothing of this thread's may still be on its way to shared memory when the CTA ends
                if (nq > 0) mbar_wait_own<1>(bar(L::B_Q_FULL), (nq - 1) & 1);
                for (int i = max(0, nk - NSK); i < nk; ++i) mbar_wait_own<1>(bar(L::B_K_FULL + i % NSK), (i / NSK) & 1);
            }
        } else if (warp == kLoadV) {
            values_ready();
            if (lane == 0 && ok) {
                int nv = 0;
                for (int u = 0;; ++u) {
                    UnitInfo x;
                    ok = unit(u, x);
                    if (!ok || x.n < 0) break;
                    unit_read(u, true);
                    const int g = x.h / a.G;
                    for (int j = 0; j < x.n; ++j, ++nv) {
                        const int st = nv % NSV;
                        if (nv >= NSV) ok = mbar_wait<1>(bar(L::B_V_FREE + st), (nv / NSV - 1) & 1, gave_up);
                        if (!ok) break;
                        mbar_arrive_expect_tx<1>(bar(L::B_V_FULL + st), TILE);
                        for (int blk = 0; blk < NB; ++blk)
                            tma_load_3d<1>(sbase + L::OFF_V + st * TILE + blk * L::BLK, &maps.v, 64 * blk, g, x.k_base + j * BN,
                                           bar(L::B_V_FULL + st));
                    }
                    if (!ok) break;
                }
                for (int i = max(0, nv - NSV); i < nv; ++i) mbar_wait_own<1>(bar(L::B_V_FULL + i % NSV), (i / NSV) & 1);
            }
        } else if (ok) {
            // The issuing warps, all lanes: trip counts and addresses come out of warp-wide reductions,
            // which leave them in uniform registers; a product whose operands are in the lanes' registers
            // costs more time to issue than to run.
            const uint32_t tb = __reduce_max_sync(0xFFFFFFFFu, tmem);
            int t = 0, nq = 0;  // tiles; units with keys
            for (int u = 0;; ++u) {
                UnitInfo x;
                ok = __all_sync(0xFFFFFFFFu, unit(u, x));
                if (!ok) break;
                const int n = __reduce_max_sync(0xFFFFFFFFu, x.n);
                __syncwarp();
                unit_read(u, lane == 0);
                if (n < 0) break;
                if (n == 0) continue;
                if (warp == kScores) {
                    constexpr uint32_t ID_S = idesc_bf16(BM, BN, false);
                    ok = wait_all(L::B_Q_FULL, nq & 1);
                    const uint32_t qd = desc_lo(sbase + L::OFF_Q, 16);
                    for (int j = 0; j < n && ok; ++j, ++t) {
                        const int st = t % NSK;
                        ok = wait_all(L::B_K_FULL + st, (t / NSK) & 1);
                        if (!L::OVER)
                            ok = ok && wait_all(L::B_S_GO, t & 1);
                        else if (t > 0)
                            ok = ok && wait_all(L::B_PV_DONE, (t - 1) & 1);
                        if (!ok) break;
                        const uint32_t kd = desc_lo(sbase + L::OFF_K + st * TILE, 16);
                        if (elect_one()) {
#pragma unroll
                            for (int ks = 0; ks < D / 16; ++ks)
                                tc_mma_ss<1>(tb, qd + dstep((ks >> 2) * L::BLK + (ks & 3) * 32), kd + dstep((ks >> 2) * L::BLK + (ks & 3) * 32), ID_S, ks > 0);
                            tc_commit<1>(bar(L::B_S_FULL));
                            tc_commit<1>(bar(L::B_K_FREE + st));
                            if (j == n - 1) tc_commit<1>(bar(L::B_Q_FREE));
                        }
                        __syncwarp();
                    }
                } else {
                    constexpr uint32_t ID_O = idesc_f16(BM, D, true);
                    for (int j = 0; j < n && ok; ++j, ++t) {
                        const int st = t % NSV;
                        ok = wait_all(L::B_V_FULL + st, (t / NSV) & 1) && wait_all(L::B_P_GO, t & 1);
                        if (!ok) break;
                        const uint32_t vd = desc_lo(sbase + L::OFF_V + st * TILE, L::BLK);
                        if (elect_one()) {
#pragma unroll
                            for (int ks = 0; ks < BN / 16; ++ks)
                                tc_mma_ts<1>(tb + L::T_O, tb + L::T_P + 8 * ks, vd + dstep(ks * 2048), ID_O, ks > 0 || j > 0);
                            tc_commit<1>(bar(L::B_PV_DONE));
                            tc_commit<1>(bar(L::B_V_FREE + st));
                        }
                        __syncwarp();
                    }
                }
                if (!ok) break;
                ++nq;
            }
            // every commit of this warp has arrived before the CTA ends (after a wait that gave up, those
            // of the tiles issued)
            if (lane == 0 && t > 0) {
                const int done = warp == kScores ? L::B_S_FULL : L::B_PV_DONE, free = warp == kScores ? L::B_K_FREE : L::B_V_FREE;
                const int ring = warp == kScores ? NSK : NSV;
                mbar_wait_own<1>(bar(done), (t - 1) & 1);
                for (int i = max(0, t - ring); i < t; ++i) mbar_wait_own<1>(bar(free + i % ring), (i / ring) & 1);
                if (warp == kScores && nq > 0) mbar_wait_own<1>(bar(L::B_Q_FREE), (nq - 1) & 1);
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(L::SOFTMAX_REGS));
        const int r = threadIdx.x;  // TMEM lane, row of the tile
        const uint32_t lane_off = (uint32_t)(warp * 32) << 16;
        const uint32_t t_s = tmem + lane_off, t_p = tmem + L::T_P + lane_off, t_o = tmem + L::T_O + lane_off;
        unsigned char *const stage = smem + L::OFF_OUT + warp * (L::BLK / kGroupWarps);
        const float sc = a.scale_log2;
        int t = 0;           // tiles
        bool there = false;  // the next scores, seen under the last exponentials: a poll takes 200 cycles and more even if they are
        if (!L::OVER && lane == 0) mbar_arrive(bar(L::B_S_GO));
        values_ready();
        bool left = false;  // units of whose rows some are to be computed from the inputs as given
        for (int u = 0; ok; ++u) {
            UnitInfo x;
            ok = __all_sync(0xFFFFFFFFu, unit(u, x));
            if (!ok || x.n < 0) break;
            __syncwarp();
            unit_read(u, lane == 0);
            float v_top;  // (on its way from here on: it is asked for at the unit's end; undefined without keys)
            asm volatile("ld.global.f32 %0, [%1];" : "=f"(v_top) : "l"(a.v_top + x.top));
            const int last_key = x.row + r + x.shift, warp_sees = x.row + warp * 32 + x.shift;
            float l = 0.f, m = -INFINITY, far = 0.f, top = -INFINITY;  // row sum, reference, its largest magnitude, largest score
            for (int j = 0; j < x.n; ++j, ++t) {
                // (after a wait that gave up the loop runs on without waiting: fewer branches in it)
                if (!__all_sync(0xFFFFFFFFu, there) && ok) ok = wait_all(L::B_S_FULL, t & 1);
                tc_fence_after();
                uint32_t su[2][64];
                tmem_issue64(t_s, su[0]);
                tmem_issue64(t_s + 64, su[1]);
                tmem_wait_ld();
                pin64(su[0]);
                pin64(su[1]);
                if (!L::OVER) {
                    tc_fence_before();
                    __syncwarp();
                    mbar_arrive_if(lane == 0, bar(L::B_S_GO));
                }
                float sv[BN];
#pragma unroll
                for (int e = 0; e < BN; ++e) sv[e] = __uint_as_float(su[e >> 6][e & 63]);
                if (warp_sees < j * BN + BN - 1) {
                    uint32_t cw[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) cw[e] = causal_word(last_key - j * BN, e);
#pragma unroll
                    for (int e = 0; e < BN; ++e) drop_unless(sv[e], cw[e >> 5], 1u << (e & 31));
                }
                const float mx = __fmul_rn(row_max(sv), sc);
                const bool upd = mx > m + kLazyLog2;
                const bool scale_o = upd && m != -INFINITY;
                const bool any_scale = __any_sync(0xFFFFFFFFu, scale_o);
                const float al = scale_o ? exp2f(m - mx) : 1.f;
                l *= al;
                m = upd ? mx : m;
                const float mu = m == -INFINITY ? 0.f : m;
                far = fmaxf(far, fabsf(mu));
                top = fmaxf(top, mx);
                uint32_t hw[BN / 2];
                float sum = weights_of<0, 96>(sv, sc, mu, hw);
                // polled here, the answers are there when the weights are
                bool settled = true;
                if (!L::OVER) {
                    settled = j == 0 || mbar_test<1>(bar(L::B_PV_DONE), (t - 1) & 1);
                    there = mbar_test<1>(bar(L::B_S_FULL), (t + 1) & 1);
                }
                l += sum + weights_of<96, BN>(sv, sc, mu, hw);
                // P's buffer is free and O has settled once the last value product is done (where P takes
                // the scores' place, the scores were computed after that; a unit's first tile: waited for
                // at the end of the last unit)
                if (!L::OVER && !__all_sync(0xFFFFFFFFu, settled) && ok) ok = wait_all(L::B_PV_DONE, (t - 1) & 1);
                tc_fence_after();
                if (any_scale) {
#pragma unroll 1
                    for (int c0 = 0; c0 < D; c0 += 32) {
                        float ov[32];
                        uint32_t ow[32];
                        tmem_ld32(t_o + c0, ov);
#pragma unroll
                        for (int e = 0; e < 32; ++e) ow[e] = __float_as_uint(ov[e] * al);
                        tmem_st32(t_o + c0, ow);
                    }
                    tmem_wait_st();
                }
                tmem_st32(t_p, hw);
                tmem_st32(t_p + 32, hw + 32);
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                mbar_arrive_if(lane == 0, bar(L::B_P_GO));
            }
            if (ok && x.n > 0) ok = wait_all(L::B_PV_DONE, (t - 1) & 1);
            if (!ok) break;
            const bool too_far = __any_sync(0xFFFFFFFFu, far > kFarLog2 && far < INFINITY);
            if (lane == 0) a.far[x.id * kGroupWarps + warp] = too_far;
            if (r < x.q_len - x.row) {
                if (too_far)
                    store_top(a, x.h, x.q_base + x.row + r, top);
                else
                    store_row(a, x.h, x.q_base + x.row + r, m - kAboveLog2, l);
            }
            if (too_far || (x.n > 0 && !(v_top < INFINITY))) {
                left = true;
                tc_fence_before();
                continue;
            }
            const int w0 = x.row + 32 * warp, rows = x.q_len - w0;  // the warp's first row, and how many it has (or more than 32)
            if (rows <= 0) continue;
            TOut *out = reinterpret_cast<TOut *>(a.out) + ((int64_t)(x.q_base + w0) * a.Hq + x.h) * D;
            const float inv = l == 0.f ? 0.f : pow2i(value_exp(v_top)) / l;
            constexpr int OC = 128 / (int)sizeof(TOut);  // columns that pass through the warp's 4 KB at a time
#pragma unroll
            for (int c0 = 0; c0 < D; c0 += OC) {
                // the last copy out of the place has read it
                if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                __syncwarp();
                if (x.n > 0) {
                    stage_out<OC, TOut>(stage, t_o + c0, inv);
                } else {  // rows without a key: zeros
                    for (int e = lane; e < 256; e += 32) reinterpret_cast<uint4 *>(stage)[e] = make_uint4(0u, 0u, 0u, 0u);
                }
                if (rows >= 32) {
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) {
                        asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(
                                         reinterpret_cast<uint64_t>(&maps.out)),
                                     "r"(c0), "r"(x.h), "r"(x.q_base + w0), "r"(smem_u32(stage))
                                     : "memory");
                        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                    }
                } else {
                    __syncwarp();
                    rows_out<OC, TOut>(stage, out + c0, (int64_t)a.Hq * D, rows);
                }
            }
            tc_fence_before();  // (O has been read before the next P is announced)
        }
        // (after everything else: they take far longer than a wait of another role may; the rings are free
        // by now, as this warp has seen the end of every product that read them)
        static_assert(kGroupWarps * kGivenFloats<D> * 4 <= L::OFF_OUT, "the rings hold every warp's part");
        __syncwarp();
        if (ok && left) units_as_given<D, TOut>(a, warp, reinterpret_cast<float *>(smem) + warp * kGivenFloats<D>);
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    if (!ok) atomicOr(&g_ris_packed_error, 2u);
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == kScores) tmem_dealloc<1, L::COLS>(tmem);
}

// ---------------------------------------------------------------- values as fp16
// Two passes over V ahead of the attention, a CTA per (run of a sequence's keys, KV head). A row sees keys
// of its own sequence and KV head only, so the scale is theirs: nothing that another prompt or head holds
// takes bits from these. Within them fp16 holds a key's values to 2^-12 of its own largest (what P's
// rounding costs) where the keys' largest values lie within 2^26 of one another. Where they do not (a key
// that most rows do not see may be that large), or are not finite, the rows are computed from the values as
// given.
constexpr int kPrepThreads = 256, kPrepWarps = kPrepThreads / 32, kMostSpan = 26;
// the pieces (16 bytes) of one head of a run's keys: this thread's piece of every kRows-th key from its
// first one
template <int D>
struct HeadPieces {
    static constexpr int P = D / 8, kRows = kPrepThreads / P, kAhead = kPackKeys / kRows;  // (a short run's pieces at once)
    const __nv_bfloat16 *v;
    int64_t stride;
    int n, row;
    __device__ __forceinline__ HeadPieces(const PackedArgs &a, const PackRun &run, int head)
        : stride(a.v_stride), n(run.n), row(threadIdx.x / P)
    {
        v = reinterpret_cast<const __nv_bfloat16 *>(a.v) + (int64_t)run.first * stride + head * D + (threadIdx.x % P) * 8;
    }
    __device__ __forceinline__ uint4 load(int i) const
    {
        return i + row < n ? *reinterpret_cast<const uint4 *>(v + (int64_t)(i + row) * stride) : make_uint4(0u, 0u, 0u, 0u);
    }
};
// part[head][run] = the largest magnitude of the run's values (upper half, bf16 without the sign, so that
// an infinity or NaN wins) and the smallest of its keys' largest ones that is not zero (lower half, 0xFFFF:
// every key is zero)
template <int D>
__global__ void __launch_bounds__(kPrepThreads) k_values_bounds(const PackedArgs a, uint32_t *part)
{
    using V = HeadPieces<D>;
    const V p(a, a.runs[blockIdx.x], blockIdx.y);
    after_last();
    uint32_t most = 0u, least = 0xFFFFFFFFu;
    for (int i = 0; i < p.n; i += V::kAhead * V::kRows) {
        uint4 x[V::kAhead];
#pragma unroll
        for (int e = 0; e < V::kAhead; ++e) x[e] = p.load(i + e * V::kRows);
#pragma unroll
        for (int e = 0; e < V::kAhead; ++e) {
            const uint32_t w[4] = {x[e].x, x[e].y, x[e].z, x[e].w};
            uint32_t m = 0u;
#pragma unroll
            for (int c = 0; c < 4; ++c) m = max(m, max((w[c] << 16) & 0x7FFFFFFFu, w[c] & 0x7FFF0000u));
#pragma unroll
            for (int o = 1; o < V::P; o <<= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
            most = max(most, m);
            least = min(least, m == 0u ? 0xFFFFFFFFu : m);
        }
    }
    most = __reduce_max_sync(0xFFFFFFFFu, most);
    least = __reduce_min_sync(0xFFFFFFFFu, least);
    __shared__ uint2 red[kPrepWarps];
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = make_uint2(most, least);
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kPrepWarps; ++w) {
            most = max(most, red[w].x);
            least = min(least, red[w].y);
        }
        part[(int64_t)blockIdx.y * a.n_runs + blockIdx.x] = most | (least >> 16);
    }
}
// v16 = fp16(v 2^-E), E from the parts of the sequence's runs, and top[seq][head] as v_top. A programmatic
// dependent of the kernel above; the attention is one of this kernel, allowed to start once every CTA here
// knows that nothing before this call is still running.
template <int D>
__global__ void __launch_bounds__(kPrepThreads) k_values_f16(const PackedArgs a, const uint32_t *part, float *top, __half *v16)
{
    using V = HeadPieces<D>;
    const PackRun run = a.runs[blockIdx.x];
    const int head = blockIdx.y;
    const V p(a, run, head);
    uint4 x[V::kAhead];
#pragma unroll
    for (int e = 0; e < V::kAhead; ++e) x[e] = p.load(e * V::kRows);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    uint32_t most = 0u, least = 0xFFFFu;
    for (int i = run.run0 + (int)threadIdx.x; i < run.run1; i += kPrepThreads) {
        const uint32_t w = part[(int64_t)head * a.n_runs + i];
        most = max(most, w & 0xFFFF0000u);
        least = min(least, w & 0xFFFFu);
    }
    most = __reduce_max_sync(0xFFFFFFFFu, most);
    least = __reduce_min_sync(0xFFFFFFFFu, least);
    __shared__ uint2 red[kPrepWarps];
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = make_uint2(most, least);
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kPrepWarps; ++w) {
        most = max(most, red[w].x);
        least = min(least, red[w].y);
    }
    const bool as_given = most >= 0x7F800000u || (least != 0xFFFFu && (int)(most >> 23) - (int)(least >> 7) > kMostSpan);
    if ((int)blockIdx.x == run.run0 && threadIdx.x == 0) top[(int64_t)run.seq * a.Hkv + head] = as_given ? INFINITY : __uint_as_float(most);
    // (zeros where v16 is not to be used: a tile at a sequence's end reaches into the next one's, under
    // weights of 0)
    const float s = as_given ? 0.f : pow2i(-value_exp(__uint_as_float(most)));
    __half *out = v16 + ((int64_t)run.first * a.Hkv + head) * D + (threadIdx.x % V::P) * 8;
    for (int i = 0;;) {
#pragma unroll
        for (int e = 0; e < V::kAhead; ++e) {
            const uint32_t w[4] = {x[e].x, x[e].y, x[e].z, x[e].w};
            uint32_t y[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const __half2 hv = __floats2half2_rn(__uint_as_float(w[c] << 16) * s, __uint_as_float(w[c] & 0xFFFF0000u) * s);
                y[c] = as_given ? 0u : *reinterpret_cast<const uint32_t *>(&hv);
            }
            const int r = i + e * V::kRows + p.row;
            if (r < p.n) *reinterpret_cast<uint4 *>(out + (int64_t)r * a.Hkv * D) = make_uint4(y[0], y[1], y[2], y[3]);
        }
        i += V::kAhead * V::kRows;
        if (i >= p.n) break;
#pragma unroll
        for (int e = 0; e < V::kAhead; ++e) x[e] = p.load(i + e * V::kRows);
    }
}

// ---------------------------------------------------------------- key weights
// What each key got from the last weight_rows rows of its sequence: w_j = sum over those rows i and the
// heads of its KV head of 2^(s_ij - m_i) / l_i, with the maxima and sums that the attention left. One CTA
// per (128 keys, KV head) holds the keys as the A operand and runs S^T = K Q^T over the group's heads and
// chunks of 64 rows: a thread owns a key (a TMEM lane), so the sum over rows stays in its register. Bounded
// by the latency of a few steps per CTA: 17 us for the last 64 rows of 9 prompts, 16,233 keys and 32 / 4
// heads of 64, whose exponentials alone take 3.6 (issue slots 34 % busy).
//
//   warps 0-3  one thread per key; warp 4 (TMA) the keys, then chunks of rows into a ring; warp 5 the products
template <int DT>
struct LayW {
    static constexpr int RC = 64, NQ = 3, NB = DT / 64;    // rows of a chunk, ring stages, 64-column blocks
    static constexpr int K_BLK = BN * 128, Q_BLK = RC * 128, Q_STAGE = NB * Q_BLK;
    static constexpr int NST = 4;                          // chunks of row statistics, a warp's own, in flight or in use
    static constexpr int OFF_K = 0, OFF_Q = OFF_K + NB * K_BLK, OFF_STAT = OFF_Q + NQ * Q_STAGE;  // float2 [4][NST][RC]
    static constexpr int OFF_BARS = OFF_STAT + 4 * NST * RC * 8, OFF_TMEM = OFF_BARS + 128, BYTES = OFF_TMEM + 16;
    static constexpr int B_K_FULL = 0, B_Q_FULL = 1, B_Q_FREE = B_Q_FULL + NQ, B_S_FULL = B_Q_FREE + NQ, B_S_FREE = B_S_FULL + 2,
                         NBAR = B_S_FREE + 2;
    static constexpr uint32_t COLS = 2 * RC;
};
constexpr int kWeightThreads = 192;

template <int DT>
__global__ void __launch_bounds__(kWeightThreads, DT == 64 ? 4 : 2) k_packed_weights_tc(const PackedArgs a, const __grid_constant__ PackedMaps maps)
{
    using L = LayW<DT>;
    constexpr int RC = L::RC, NQ = L::NQ, NB = L::NB, NST = L::NST;
    extern __shared__ __align__(1024) unsigned char smem[];
    uint32_t &tmem_base_sh = *reinterpret_cast<uint32_t *>(smem + L::OFF_TMEM);
    const uint32_t sbase = smem_u32(smem);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const unsigned int *const gave_up = &g_ris_packed_error;
    after_last();
    const PackItem it = a.key_items[blockIdx.x];
    const int g = blockIdx.y, shift = it.k_len - it.q_len;
    // rows that count and see the item's first key
    const int first = max(max(0, it.q_len - a.weight_rows), it.row - shift);
    const int chunks = first < it.q_len ? (it.q_len - first + RC - 1) / RC : 0, steps = chunks * a.G;
    const int j = it.row + (int)threadIdx.x;  // this thread's key (warps 0-3)
    if (steps == 0) {
        if (threadIdx.x < BN && j < it.k_len) a.key_weight[(int64_t)g * a.k_total + it.k_base + j] = 0.f;
        return;
    }
    auto bar = [&](int i) { return sbase + (uint32_t)(L::OFF_BARS + 8 * i); };
    if (warp == 4) {
        if (lane < L::NBAR) {
            mbar_init(bar(lane), lane >= L::B_S_FREE ? 4 : 1);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
    } else if (warp == 5) {
        tmem_alloc<1, L::COLS>(smem_u32(&tmem_base_sh));
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_base_sh;
    bool ok = (sbase & 1023u) == 0u;
    if (warp == 4) {
        if (lane == 0 && ok) {
            mbar_arrive_expect_tx<1>(bar(L::B_K_FULL), NB * L::K_BLK);
            for (int blk = 0; blk < NB; ++blk)
                tma_load_3d<1>(sbase + L::OFF_K + blk * L::K_BLK, &maps.k, 64 * blk, g, it.k_base + it.row, bar(L::B_K_FULL));
            int n = 0;
            for (int s = 0; s < steps && ok; ++s) {
                const int st = s % NQ, h = g * a.G + s / chunks, row = it.q_base + first + s % chunks * RC;
                if (s >= NQ) ok = mbar_wait<1>(bar(L::B_Q_FREE + st), (s / NQ - 1) & 1, gave_up);
                if (!ok) break;
                mbar_arrive_expect_tx<1>(bar(L::B_Q_FULL + st), L::Q_STAGE);
                for (int blk = 0; blk < NB; ++blk)
                    tma_load_3d<1>(sbase + L::OFF_Q + st * L::Q_STAGE + blk * L::Q_BLK, &maps.q, 64 * blk, h, row, bar(L::B_Q_FULL + st));
                n = s + 1;
            }
            mbar_wait_own<1>(bar(L::B_K_FULL), 0);
            for (int s = max(0, n - NQ); s < n; ++s) mbar_wait_own<1>(bar(L::B_Q_FULL + s % NQ), (s / NQ) & 1);
        }
    } else if (warp == 5) {
        constexpr uint32_t ID = idesc_bf16(BN, RC, false);
        const uint32_t tb = __reduce_max_sync(0xFFFFFFFFu, tmem);  // (into a uniform register)
        auto wait_all = [&](int i, int parity) -> bool {
            const bool got = __all_sync(0xFFFFFFFFu, mbar_wait<1>(bar(i), parity, gave_up));
            tc_fence_after();
            return got;
        };
        if (ok) ok = wait_all(L::B_K_FULL, 0);
        int n = 0;
        for (int s = 0; s < steps && ok; ++s) {
            const int st = s % NQ, b = s & 1;
            ok = wait_all(L::B_Q_FULL + st, (s / NQ) & 1);
            if (ok && s >= 2) ok = wait_all(L::B_S_FREE + b, (s / 2 - 1) & 1);
            if (!ok) break;
            const uint32_t kd = desc_lo(sbase + L::OFF_K, 16), qd = desc_lo(sbase + L::OFF_Q + st * L::Q_STAGE, 16);
            if (elect_one()) {
#pragma unroll
                for (int ks = 0; ks < DT / 16; ++ks)
                    tc_mma_ss<1>(tb + b * RC, kd + dstep((ks >> 2) * L::K_BLK + (ks & 3) * 32), qd + dstep((ks >> 2) * L::Q_BLK + (ks & 3) * 32),
                                 ID, ks > 0);
                tc_commit<1>(bar(L::B_S_FULL + b));
                tc_commit<1>(bar(L::B_Q_FREE + st));
            }
            __syncwarp();
            n = s + 1;
        }
        // every commit has arrived before the CTA ends
        if (lane == 0) {
            for (int s = max(0, n - 2); s < n; ++s) mbar_wait_own<1>(bar(L::B_S_FULL + (s & 1)), (s / 2) & 1);
            for (int s = max(0, n - NQ); s < n; ++s) mbar_wait_own<1>(bar(L::B_Q_FREE + s % NQ), (s / NQ) & 1);
        }
    } else {
        float2 *const st_sh = reinterpret_cast<float2 *>(smem + L::OFF_STAT) + warp * NST * RC;
        const float sc = a.scale_log2;
        const uint32_t lane_off = (uint32_t)(warp * 32) << 16;
        float w = 0.f;
        // the maxima and 1 / sums of step s's rows, zeros past the last row
        auto stats = [&](int s) {
            if (s < steps) {
                const int i0 = first + s % chunks * RC;
                const float2 *p = a.row_stat + (int64_t)(g * a.G + s / chunks) * a.q_total + it.q_base;
#pragma unroll
                for (int e = lane; e < RC; e += 32)
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(smem_u32(st_sh + s % NST * RC + e)),
                                 "l"(p + min(i0 + e, it.q_len - 1)), "r"(i0 + e < it.q_len ? 8 : 0)
                                 : "memory");
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        for (int s = 0; s < NST - 1; ++s) stats(s);
        for (int s = 0; s < steps && ok; ++s) {
            asm volatile("cp.async.wait_group %0;" ::"n"(NST - 2) : "memory");
            __syncwarp();  // step s's are there for every lane, and every lane is done with those of step s - 1
            stats(s + NST - 1);
            const float2 *const st = st_sh + s % NST * RC;
            ok = __all_sync(0xFFFFFFFFu, mbar_wait<1>(bar(L::B_S_FULL + (s & 1)), (s / 2) & 1, gave_up));
            if (!ok) break;
            tc_fence_after();
            const int i0 = first + s % chunks * RC;
            const int from = j - shift - i0;   // first row of the chunk that sees this thread's key
            const int rows = it.q_len - i0;    // rows of the chunk
            const bool whole = it.row + warp * 32 + 31 - shift <= i0 && rows >= RC;
            // (a far row's maximum was rounded as a product, the others' sums came from exponents rounded once)
            const bool far = __any_sync(0xFFFFFFFFu, fmaxf(fabsf(st[lane].x), fabsf(st[lane + 32].x)) > kFarLog2);
            static_assert(RC == 64, "two rows to a lane");
            float part[4] = {};
            auto add = [&](auto far_c) {
                auto weight = [&](float x, float m) { return ex2(decltype(far_c)::value ? __fmul_rn(x, sc) - m : fmaf(x, sc, -m)); };
#pragma unroll
                for (int half = 0; half < RC; half += 32) {
                    float sv[32];
                    tmem_ld32(tmem + (s & 1) * RC + lane_off + half, sv);
                    if (half == RC - 32) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0 && s + 2 < steps) mbar_arrive(bar(L::B_S_FREE + (s & 1)));
                    }
                    if (whole) {
#pragma unroll
                        for (int e = 0; e < 32; e += 2) {
                            const float4 ml = *reinterpret_cast<const float4 *>(&st[half + e]);
                            part[e & 2] = fmaf(weight(sv[e], ml.x), ml.y, part[e & 2]);
                            part[(e & 2) + 1] = fmaf(weight(sv[e + 1], ml.z), ml.w, part[(e & 2) + 1]);
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; ++e) {
                            const float2 ml = st[half + e];
                            const float p = weight(sv[e], ml.x);
                            if (half + e >= from && half + e < rows) part[e & 3] = fmaf(p, ml.y, part[e & 3]);
                        }
                    }
                }
            };
            if (far)
                add(std::true_type{});
            else
                add(std::false_type{});
            w += (part[0] + part[1]) + (part[2] + part[3]);
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        if (ok && j < it.k_len) a.key_weight[(int64_t)g * a.k_total + it.k_base + j] = w;
    }
    if (!ok) atomicOr(&g_ris_packed_error, 2u);
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 5) tmem_dealloc<1, L::COLS>(tmem);
}

// ---------------------------------------------------------------- host side
// n tokens of H heads of D values, `stride` elements from token to token, viewed as 3D (d, head, token); box =
// 128 bytes of d x 1 head x `rows` tokens.
bool make_map(CUtensorMap *m, CUtensorMapDataType type, const void *base, int64_t n, int H, int64_t stride, int rows, int D)
{
    auto fn = encode_fn();
    if (fn == nullptr) return false;
    const int size = type == CU_TENSOR_MAP_DATA_TYPE_FLOAT32 ? 4 : 2;
    cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)H, (cuuint64_t)n};
    cuuint64_t strides[2] = {(cuuint64_t)D * size, (cuuint64_t)stride * size};
    cuuint32_t box[3] = {(cuuint32_t)(128 / size), 1, (cuuint32_t)rows};
    cuuint32_t estr[3] = {1, 1, 1};
    return fn(m, type, 3, const_cast<void *>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
constexpr CUtensorMapDataType kBf16 = CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, kF16 = CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
                              kF32 = CU_TENSOR_MAP_DATA_TYPE_FLOAT32;

using TileKernel = void (*)(PackedArgs, PackedMaps);

// Once per kernel: its shared memory, and that its launch has the `regs` registers a thread that the
// softmax threads' setmaxnreg would wait for.
cudaError_t prepare(TileKernel kern, int bytes, int regs)
{
    cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    cudaFuncAttributes fa;
    if (e == cudaSuccess) e = cudaFuncGetAttributes(&fa, kern);
    return e != cudaSuccess ? e : (fa.numRegs + 7) / 8 * 8 < regs ? cudaErrorInvalidConfiguration : cudaSuccess;
}

template <typename TOut>
cudaError_t launch_clusters(const PackedArgs &a, const PackedMaps &maps, cudaStream_t s)
{
    static_assert(Lay128::BYTES > 232448 / 2, "one CTA per SM, as it holds all TMEM columns");
    static Once once;
    const cudaError_t ready = once([] { return prepare(k_packed128<TOut>, Lay128::BYTES, kRegs); });
    if (ready != cudaSuccess) return ready;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((int64_t)a.n_items * ((a.G & 1) == 0 ? a.Hq / 2 : a.Hq) * 2));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = Lay128::BYTES;
    cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = 2;
    at[1].val.clusterDim.y = 1;
    at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, k_packed128<TOut>, a, maps);
    note_launch();
    return e != cudaSuccess ? e : cudaGetLastError();
}

template <int D, typename TOut>
cudaError_t launch_rows(const PackedArgs &a, const PackedMaps &maps, cudaStream_t s)
{
    using L = LayRows<D>;
    static Once once;
    const cudaError_t ready = once([] { return prepare(k_packed_rows<D, TOut>, L::BYTES, L::REGS); });
    if (ready != cudaSuccess) return ready;
    const int64_t units = (int64_t)a.n_items * a.Hq;
    return launch_chained(k_packed_rows<D, TOut>, dim3((unsigned)std::min<int64_t>(units, 2 * 152)), dim3(L::THREADS), L::BYTES, s, a, maps);
}

}  // namespace

// scratch: the bounds of the runs, the largest magnitudes, the units' marks, the values
static size_t scratch_part(const PackedArgs &a) { return (sizeof(uint32_t) * a.n_runs * a.Hkv + 255) & ~size_t(255); }
static size_t scratch_top(const PackedArgs &a) { return (sizeof(float) * a.n_seqs * a.Hkv + 255) & ~size_t(255); }
static size_t scratch_far(const PackedArgs &a) { return ((size_t)a.n_items * a.Hq * kGroupWarps + 255) & ~size_t(255); }
size_t packed_scratch_bytes(const PackedArgs &a, int32_t head_dim)
{
    return scratch_part(a) + scratch_top(a) + scratch_far(a) + (size_t)a.k_total * a.Hkv * head_dim * 2;
}

cudaError_t launch_packed_tiles(PackedArgs a, int D, int out_dtype, bool clusters, void *scratch, cudaStream_t s)
{
    char *const mem = static_cast<char *>(scratch);
    uint32_t *const part = reinterpret_cast<uint32_t *>(mem);
    float *const top = reinterpret_cast<float *>(mem + scratch_part(a));
    a.far = reinterpret_cast<uint8_t *>(mem + scratch_part(a) + scratch_top(a));
    __half *const v16 = reinterpret_cast<__half *>(mem + scratch_part(a) + scratch_top(a) + scratch_far(a));
    a.v_top = top;
    if (a.n_runs > 0) {
        const dim3 grid((unsigned)a.n_runs, (unsigned)a.Hkv);
        cudaError_t e = launch_chained(D == 128 ? k_values_bounds<128> : k_values_bounds<64>, grid, dim3(kPrepThreads), 0, s, a, part);
        if (e != cudaSuccess) return e;
        e = launch_chained(D == 128 ? k_values_f16<128> : k_values_f16<64>, grid, dim3(kPrepThreads), 0, s, a, part, top, v16);
        if (e != cudaSuccess) return e;
    }
    alignas(64) PackedMaps maps;
    const CUtensorMapDataType out_type = out_dtype == RIS_F32 ? kF32 : kBf16;
    if (!make_map(&maps.q, kBf16, a.q, a.q_total, a.Hq, a.q_stride, BM, D) ||
        !make_map(&maps.out, out_type, a.out, a.q_total, a.Hq, (int64_t)a.Hq * D, 32, D))
        return cudaErrorInvalidValue;
    // (without keys no box of k or v is ever asked for: any valid map does)
    if (a.k_total == 0)
        maps.k = maps.v = maps.q;
    else if (!make_map(&maps.k, kBf16, a.k, a.k_total, a.Hkv, a.k_stride, clusters ? Lay128::KROWS : BN, D) ||
             !make_map(&maps.v, kF16, v16, a.k_total, a.Hkv, (int64_t)a.Hkv * D, BN, D))
        return cudaErrorInvalidValue;
    if (clusters) return out_dtype == RIS_F32 ? launch_clusters<float>(a, maps, s) : launch_clusters<__nv_bfloat16>(a, maps, s);
    if (D == 128) return out_dtype == RIS_F32 ? launch_rows<128, float>(a, maps, s) : launch_rows<128, __nv_bfloat16>(a, maps, s);
    return out_dtype == RIS_F32 ? launch_rows<64, float>(a, maps, s) : launch_rows<64, __nv_bfloat16>(a, maps, s);
}

cudaError_t launch_packed_weights_tc(const PackedArgs &a, int D, cudaStream_t s)
{
    alignas(64) PackedMaps maps;
    if (a.q_total == 0)
        maps = PackedMaps{};  // no rows: every CTA writes zeros
    else if (!make_map(&maps.q, kBf16, a.q, a.q_total, a.Hq, a.q_stride, LayW<128>::RC, D) ||
             !make_map(&maps.k, kBf16, a.k, a.k_total, a.Hkv, a.k_stride, BN, D))
        return cudaErrorInvalidValue;
    else
        maps.v = maps.k;
    const dim3 grid((unsigned)a.n_key_items, (unsigned)a.Hkv);
    if (D == 128) {
        static Once once;
        const cudaError_t ready = once([] { return prepare(k_packed_weights_tc<128>, LayW<128>::BYTES, 0); });
        if (ready != cudaSuccess) return ready;
        return launch_chained(k_packed_weights_tc<128>, grid, dim3(kWeightThreads), LayW<128>::BYTES, s, a, maps);
    } else {
        // 52 KB where 49 would do: four CTAs to an SM; five would ask for more TMEM columns than there are
        constexpr int bytes = 52 << 10;
        static_assert(bytes >= LayW<64>::BYTES, "");
        static Once once;
        const cudaError_t ready = once([] { return prepare(k_packed_weights_tc<64>, bytes, 0); });
        if (ready != cudaSuccess) return ready;
        return launch_chained(k_packed_weights_tc<64>, grid, dim3(kWeightThreads), bytes, s, a, maps);
    }
}

cudaError_t packed_error_word(unsigned int **p) { return cudaGetSymbolAddress(reinterpret_cast<void **>(p), g_ris_packed_error); }

}  // namespace ris
