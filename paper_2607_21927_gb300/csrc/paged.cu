// A cache in pages: writing rows into it, the plan of an attention call whose sequences have several row
// tiles, the join of row tiles that several CTAs worked on, and attention in fp32 (the FP32 pipe; inputs
// never pass through a narrower product). bf16: attn_paged.cu.
#include <cuda_bf16.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "attn_common.cuh"
#include "attn_paged.cuh"

namespace ris {

// Device error word of this file (bit 1: a token or key outside the pages); read by ris_device_status.
__device__ unsigned int g_ris_paged_error;

namespace {

using namespace paged;

// ---------------------------------------------------------------- writing rows
// Threads take 16-byte pieces of a CTA's rows of k and v, all of a thread's loads before its stores. Bound by
// HBM, each row read and written once; a row's place is a chain of loads (sequence, start, page), which is
// all that a call of few rows takes.
constexpr int kAppendThreads = 256, kAppendPieces = 4;

__device__ __forceinline__ int new_length(const PagedAppendArgs &a, int b, const int32_t *start)
{
    const int64_t n = (int64_t)start[b] + a.off[b + 1] - a.off[b];
    return (int)max((int64_t)0, min(n, (int64_t)a.c.table_len << a.c.page_log2));
}

template <typename T>
__global__ void __launch_bounds__(kAppendThreads) k_paged_append(const __grid_constant__ PagedAppendArgs a)
{
    constexpr int V = 16 / (int)sizeof(T), U = kAppendPieces;
    after_last();
    const int pieces = a.c.Hkv * a.c.D / V;  // of a row
    const int64_t r0 = (int64_t)blockIdx.x * a.rows;
    const int n = (int)min((int64_t)a.rows, a.total - r0) * pieces;
    const int32_t *const start = a.start != nullptr ? a.start : a.c.length;
    for (int t0 = threadIdx.x; t0 < n; t0 += U * kAppendThreads) {
        uint4 k[U], v[U];
        int64_t at[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int t = t0 + u * kAppendThreads;
            at[u] = -1;
            if (t >= n) continue;
            const int64_t row = r0 + t / pieces;
            const int e = t % pieces * V;
            k[u] = *reinterpret_cast<const uint4 *>(reinterpret_cast<const T *>(a.k) + row * a.k_stride + e);
            v[u] = *reinterpret_cast<const uint4 *>(reinterpret_cast<const T *>(a.v) + row * a.v_stride + e);
            const int seq = a.seq_of[row];
            const int64_t slot = start[seq] + (row - a.off[seq]);
            int page = -1;
            if (slot >= 0 && slot >> a.c.page_log2 < a.c.table_len) page = page_of(a.c, seq, (int)slot);
            if (page >= 0)
                at[u] = slot_at(a.c, page, e / a.c.D, (int)slot) + e % a.c.D;
            else
                atomicOr(&g_ris_paged_error, 1u);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (at[u] >= 0) {
                *reinterpret_cast<uint4 *>(reinterpret_cast<T *>(a.c.k) + at[u]) = k[u];
                *reinterpret_cast<uint4 *>(reinterpret_cast<T *>(a.c.v) + at[u]) = v[u];
            }
    }
    // the lengths: nobody else reads or writes them where `start` is given; else only this CTA may
    if (blockIdx.x != 0 || (a.start == nullptr && gridDim.x > 1)) return;
    __syncthreads();
    for (int b = threadIdx.x; b < a.c.B; b += kAppendThreads) a.c.length[b] = new_length(a, b, start);
}

__global__ void __launch_bounds__(kAppendThreads) k_paged_lengths(const __grid_constant__ PagedAppendArgs a)
{
    after_last();
    for (int b = blockIdx.x * kAppendThreads + threadIdx.x; b < a.c.B; b += gridDim.x * kAppendThreads)
        a.c.length[b] = new_length(a, b, a.start != nullptr ? a.start : a.c.length);
}

// ---------------------------------------------------------------- the plan
// Where sequences have several row tiles: the items (sequence, row tile) and the cost of those before each.
// One CTA: 1,000 items take 3 us, ahead of an attention call of hundreds.
constexpr int kPlanThreads = 1024;

template <int KEYS>
__global__ void __launch_bounds__(kPlanThreads) k_paged_plan(const __grid_constant__ PagedAttendArgs a)
{
    __shared__ int64_t mem[kPlanThreads / 32];
    after_last();
    int64_t all, before = 0;
    for (int s0 = 0; s0 < a.c.B; s0 += kPlanThreads) {
        const int s = s0 + threadIdx.x;
        const int tiles = s < a.c.B ? (a.off[s + 1] - a.off[s] + a.tokens - 1) / a.tokens : 0;
        const int64_t at = before + block_scan<kPlanThreads>(tiles, mem, all);
        if (s < a.c.B) a.seq_items[s] = (int)at;
        before += all;
    }
    const int n = (int)before;
    __syncthreads();  // (seq_items is read by the whole block)
    before = 0;
    for (int i0 = 0; i0 < n; i0 += kPlanThreads) {
        const int i = i0 + threadIdx.x;
        int64_t cost = 0;
        if (i < n) {
            int lo = 0, hi = a.c.B - 1;  // the last sequence whose first item is at or before i
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (a.seq_items[mid] <= i)
                    lo = mid;
                else
                    hi = mid - 1;
            }
            const PagedItem it{lo, i - a.seq_items[lo]};
            a.items[i] = it;
            cost = sight_of<KEYS>(a, length_of(a, lo), a.off[lo + 1] - a.off[lo], it.tile).n + 1;
        }
        const int64_t at = before + block_scan<kPlanThreads>(cost, mem, all);
        if (i < n) a.prefix[i] = at;
        before += all;
    }
    if (threadIdx.x == 0) {
        a.prefix[n] = before;
        *a.n_items = n;
    }
}

// ---------------------------------------------------------------- the join
// out = sum_p 2^(m_p - m) O_p / sum_p 2^(m_p - m) n_p over the parts of a row, in their order, and its log-sum-exp from
// the sums l_p (n_p is l_p, or with a weight as it was rounded). CTAs (run that began the row tile, group of rows);
// W warps take every W-th part of a row and are added up in order.
constexpr int kJoinThreads = 256, kJoinWarps = kJoinThreads / 32;

template <typename T, int D, int W>
__global__ void __launch_bounds__(kJoinThreads) k_paged_join(const __grid_constant__ PagedAttendArgs a)
{
    constexpr int C = D / 32, ROWS = kJoinWarps / W;
    __shared__ float4 ml[kJoinWarps];
    __shared__ float os[kJoinWarps][D];
    after_last();
    const PagedSplit sp = a.split[blockIdx.x];
    if (sp.first < 0) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, wr = warp % W;
    const int r = blockIdx.y * ROWS + warp / W, token = r / a.block, head = r % a.block;
    const bool there = token < sp.tokens && head < sp.heads;
    float m = -INFINITY, l = 0.f, n = 0.f, o[C] = {};
    if (there) {
        auto place = [&](int c) { return (int64_t)(2 * c + (c == sp.first ? 1 : 0)) * a.part_rows + r; };
        // (a lane looks at every 32nd of the warp's parts)
        for (int c = sp.first + wr + W * lane; c <= sp.last; c += 32 * W) m = fmaxf(m, a.part_ml[place(c)].x);
        m = warp_max(m);
        const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll 4
        for (int c = sp.first + wr; c <= sp.last; c += W) {
            const float4 y = a.part_ml[place(c)];
            const float *p = a.part_o + place(c) * D + C * lane;
            float z[C];
            if constexpr (C == 4) {
                const float4 q = *reinterpret_cast<const float4 *>(p);
                z[0] = q.x, z[1] = q.y, z[2] = q.z, z[3] = q.w;
            } else {
                const float2 q = *reinterpret_cast<const float2 *>(p);
                z[0] = q.x, z[1] = q.y;
            }
            // (a part without a visible key adds nothing, whatever its product holds)
            const float f = y.y == 0.f ? 0.f : exp2f(y.x - ref);
            l = fmaf(y.y, f, l);
            n = fmaf(y.z, f, n);
#pragma unroll
            for (int e = 0; e < C; ++e) o[e] = y.y == 0.f ? o[e] : fmaf(z[e], f, o[e]);
        }
    }
    if constexpr (W > 1) {
        if (lane == 0) ml[warp] = make_float4(m, l, n, 0.f);
#pragma unroll
        for (int e = 0; e < C; ++e) os[warp][C * lane + e] = o[e];
        __syncthreads();
        if (wr != 0) return;
        for (int i = 0; i < W; ++i) m = fmaxf(m, ml[warp + i].x);
        const float ref = m == -INFINITY ? 0.f : m;
        l = n = 0.f;
#pragma unroll
        for (int e = 0; e < C; ++e) o[e] = 0.f;
        for (int i = 0; i < W; ++i) {
            const float4 y = ml[warp + i];
            if (y.y == 0.f) continue;
            const float f = exp2f(y.x - ref);
            l = fmaf(y.y, f, l);
            n = fmaf(y.z, f, n);
#pragma unroll
            for (int e = 0; e < C; ++e) o[e] = fmaf(os[warp + i][C * lane + e], f, o[e]);
        }
    }
    if (!there) return;
    const int64_t row = sp.row0 + token;
    T *out = reinterpret_cast<T *>(a.out) + (row * a.Hq + sp.head0 + head) * D + C * lane;
#pragma unroll
    for (int e = 0; e < C; ++e) {
        const float x = l == 0.f ? 0.f : o[e] / n;
        if constexpr (sizeof(T) == 4)
            out[e] = x;
        else
            out[e] = __float2bfloat16_rn(x);
    }
    if (lane == 0 && a.lse != nullptr) a.lse[(sp.head0 + head) * a.q_total + row] = (m + log2f(l)) * kLn2;
}

// ---------------------------------------------------------------- attention in fp32
// A CTA walks its run of (32 rows x 64 keys) tiles with a running maximum and sum. Keys and values come row by
// row by cp.async into a buffer each, the next keys under the value product and the next values under the
// scores. S: a 4 x 4 patch per thread, 4 elements at a time as packed pairs; the softmax over the 16 lanes
// that share a row; O += P V with a 4 x D / 16 patch, P as pairs of the same weight in shared memory. Bound by
// the FMA pipe: 4 D flops per row and key.
constexpr int BM = kPagedF32Rows, BN = kPagedF32Keys, LP = 2 * BN + 4;  // rows and keys of a tile, pitch of P
constexpr int kThreads = 4 * BM;

__device__ __forceinline__ void store4(float *p, float4 x) { *reinterpret_cast<float4 *>(p) = x; }
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
// 16 bytes to shared memory, or zeros
__device__ __forceinline__ void copy16(float *dst, const float *src, bool there)
{
    const uint32_t to = (uint32_t)__cvta_generic_to_shared(dst);
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copied_but()  // all but the last N groups
{
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// The keys (or values) of a tile that some row of the unit sees, the others as zeros, into rows of pitch
// D + 4 or D
template <int D, bool PAD>
__device__ __forceinline__ void fetch_keys(const PagedAttendArgs &a, const Unit &u, float *dst, const void *pool, int k0)
{
#pragma unroll 4
    for (int e = 0; e < BN * (D / 4) / kThreads; ++e) {
        const int t = threadIdx.x + e * kThreads, r = t / (D / 4), d = t % (D / 4) * 4, j = k0 + r;
        bool there = j < u.sight.end && (j >= u.sight.low || j < a.anchors);
        const float *src = reinterpret_cast<const float *>(pool);
        if (there) {
            const int page = page_of(a.c, u.seq, j);
            there = page >= 0;
            if (there)
                src += slot_at(a.c, page, u.kv_head, j) + d;
            else
                atomicOr(&g_ris_paged_error, 1u);
        }
        copy16(dst + r * (PAD ? D + 4 : D) + d, src, there);
    }
    copies_end();
}

template <int D>
__global__ void __launch_bounds__(kThreads, 2) k_paged_f32(const __grid_constant__ PagedAttendArgs a)
{
    constexpr int LK = D + 4, C = D / 16;  // columns of O of a thread
    extern __shared__ __align__(16) float sm[];
    float *const qs = sm, *const ks = qs + BM * LK, *const vs = ks + BN * LK, *const ps = vs + BN * D;
    __shared__ RunMem mem;
    after_last();
    const Run run = run_of<BN, kThreads>(a, blockIdx.x, mem);
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;  // rows 4 ty + i; keys tx + 16 j; columns 4 tx + 64 c
    PagedSplit split{-1};
    Walk walk(run);
    Unit u;
    while (walk.next<BN>(a, run, u)) {
        if (u.split.first >= 0) split = u.split;
        __syncthreads();  // the last unit's buffers are free
        // the query rows: token r / block, head r % block; zeros for rows that there are not
        for (int e = 0; e < BM * (D / 4) / kThreads && u.j0 < u.j1; ++e) {
            const int t = threadIdx.x + e * kThreads, r = t / (D / 4), d = t % (D / 4) * 4, tok = r / a.block, h = r % a.block;
            const bool there = tok < u.sight.tokens && h < u.heads;
            const float *q = reinterpret_cast<const float *>(a.q) + (there ? (int64_t)(u.row0 + tok) * a.q_stride + (u.head0 + h) * D + d : 0);
            copy16(qs + r * LK + d, q, there);
        }
        if (u.j0 < u.j1) {
            fetch_keys<D, true>(a, u, ks, a.c.k, BN * u.sight.tile(u.j0));
            fetch_keys<D, false>(a, u, vs, a.c.v, BN * u.sight.tile(u.j0));
        }
        int pos[4];  // of each row; one that is not there sees nothing
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 4 * ty + i, tok = r / a.block;
            pos[i] = tok < u.sight.tokens && r % a.block < u.heads ? u.sight.pos0 + tok : -1;
        }
        uint64_t o[4][C / 2] = {};
        float m[4], l[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) m[i] = -INFINITY, l[i] = 0.f;
        for (int t = u.j0; t < u.j1; ++t) {
            const int k0 = BN * u.sight.tile(t);
            const bool more = t + 1 < u.j1;
            // whether every row sees the whole tile
            const bool whole = k0 + BN - 1 <= u.sight.pos0 && (k0 + BN <= a.anchors || a.window == 0 || u.sight.pos0 + u.sight.tokens - 1 - k0 < a.window);
            copied_but<1>();  // (the values' copy may still be on its way)
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
            if (more)
                fetch_keys<D, true>(a, u, ks, a.c.k, BN * u.sight.tile(t + 1));
            else
                copies_end();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float s[4], mx = -INFINITY;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 x = f2_get(s2[i][j]);
                    s[j] = sees(a, pos[i], k0 + tx + 16 * j) ? (x.x + x.y) * a.scale_log2 : -INFINITY;
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
            copied_but<1>();  // (the next keys' copy may still be on its way)
            __syncthreads();
            // O += P V; where some row does not see the whole tile, a row takes only the keys that it sees (0 times
            // an infinity or NaN in a key's place is not 0)
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
                            if (decltype(masked)::value && !sees(a, pos[i], k0 + j + e)) continue;
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
            if (whole)
                values(std::false_type{});
            else
                values(std::true_type{});
            __syncthreads();  // the values' buffer and P's are free
            if (more)
                fetch_keys<D, false>(a, u, vs, a.c.v, BN * u.sight.tile(t + 1));
            else
                copies_end();
        }
        copied_but<0>();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float sum = l[i];
#pragma unroll
            for (int x = 8; x > 0; x >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, x);
            const int r = 4 * ty + i, tok = r / a.block, h = r % a.block;
            if (tok >= u.sight.tokens || h >= u.heads) continue;
            const int64_t row = u.row0 + tok;
            if (u.part < 0) {
                const float inv = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;  // no key: zeros; NaN stays
                float *out = reinterpret_cast<float *>(a.out) + (row * a.Hq + u.head0 + h) * D;
                if (tx == 0 && a.lse != nullptr) a.lse[(u.head0 + h) * a.q_total + row] = (m[i] + log2f(sum)) * kLn2;
#pragma unroll
                for (int c = 0; c < C / 4; ++c) {
                    const float2 x = f2_get(o[i][2 * c]), y = f2_get(o[i][2 * c + 1]);
                    store4(out + 64 * c + 4 * tx, make_float4(x.x * inv, x.y * inv, y.x * inv, y.y * inv));
                }
            } else {
                const int64_t at = (int64_t)u.part * a.part_rows + r;
                if (tx == 0) a.part_ml[at] = make_float4(m[i], sum, sum, 0.f);
#pragma unroll
                for (int c = 0; c < C / 4; ++c) {
                    const float2 x = f2_get(o[i][2 * c]), y = f2_get(o[i][2 * c + 1]);
                    store4(a.part_o + at * D + 64 * c + 4 * tx, make_float4(x.x, x.y, y.x, y.y));
                }
            }
        }
    }
    if (threadIdx.x == 0) a.split[blockIdx.x] = split;
}

template <int D>
cudaError_t launch_f32(const PagedAttendArgs &a, cudaStream_t s)
{
    constexpr int bytes = ((BM + BN) * (D + 4) + BN * D + BM * LP) * (int)sizeof(float);
    static Once once;
    const cudaError_t ready = once([] { return cudaFuncSetAttribute(k_paged_f32<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes); });
    if (ready != cudaSuccess) return ready;
    return launch_chained(k_paged_f32<D>, dim3((unsigned)a.ctas), dim3(kThreads), bytes, s, a);
}

template <typename T, int D>
cudaError_t launch_join(const PagedAttendArgs &a, cudaStream_t s)
{
    // few rows: every warp of a CTA on the parts of one row, else a row for each
    if (a.part_rows <= 32) return launch_chained(k_paged_join<T, D, kJoinWarps>, dim3((unsigned)a.ctas, (unsigned)a.part_rows), dim3(kJoinThreads), 0, s, a);
    return launch_chained(k_paged_join<T, D, 1>, dim3((unsigned)a.ctas, (unsigned)((a.part_rows + kJoinWarps - 1) / kJoinWarps)), dim3(kJoinThreads), 0, s, a);
}

}  // namespace

cudaError_t launch_paged_append(PagedAppendArgs a, int dtype, cudaStream_t s)
{
    const int pieces = a.c.Hkv * a.c.D / (dtype == RIS_F32 ? 4 : 8);
    constexpr int64_t full = kAppendThreads * kAppendPieces;  // of a CTA
    // one CTA where it can take everything, else full ones, or two on every SM
    const int64_t most = std::max<int64_t>(1, full / pieces);
    a.rows = (int)(a.total * pieces <= full ? a.total : std::min<int64_t>(most, std::max<int64_t>(1, a.total / kPagedCtas)));
    int64_t blocks = 0;
    if (a.total > 0) {
        blocks = (a.total + a.rows - 1) / a.rows;
        const cudaError_t e = dtype == RIS_F32 ? launch_chained(k_paged_append<float>, dim3((unsigned)blocks), dim3(kAppendThreads), 0, s, a)
                                               : launch_chained(k_paged_append<__nv_bfloat16>, dim3((unsigned)blocks), dim3(kAppendThreads), 0, s, a);
        if (e != cudaSuccess) return e;
    }
    if (blocks == 1 || (blocks > 0 && a.start != nullptr)) return cudaSuccess;
    if (blocks == 0 && a.start == nullptr) return cudaSuccess;
    return launch_chained(k_paged_lengths, dim3((unsigned)std::min<int64_t>(16, (a.c.B + kAppendThreads - 1) / kAppendThreads)), dim3(kAppendThreads), 0, s, a);
}

cudaError_t launch_paged_plan(const PagedAttendArgs &a, int dtype, cudaStream_t s)
{
    return launch_chained(dtype == RIS_F32 ? k_paged_plan<kPagedF32Keys> : k_paged_plan<kPagedTileKeys>, dim3(1), dim3(kPlanThreads), 0, s, a);
}

cudaError_t launch_paged_join(const PagedAttendArgs &a, int dtype, cudaStream_t s)
{
    if (dtype == RIS_F32) return a.c.D == 128 ? launch_join<float, 128>(a, s) : launch_join<float, 64>(a, s);
    return a.c.D == 128 ? launch_join<__nv_bfloat16, 128>(a, s) : launch_join<__nv_bfloat16, 64>(a, s);
}

cudaError_t launch_paged_f32(const PagedAttendArgs &a, cudaStream_t s) { return a.c.D == 128 ? launch_f32<128>(a, s) : launch_f32<64>(a, s); }

cudaError_t paged_error_word(unsigned int **p) { return cudaGetSymbolAddress(reinterpret_cast<void **>(p), g_ris_paged_error); }

}  // namespace ris
