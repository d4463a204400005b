// A cache in pages: writing rows into it, the plan of an attention call whose sequences have several row
// tiles, the join of row tiles that several CTAs worked on, and attention in fp32 (the FP32 pipe; inputs
// never pass through a narrower product). bf16: attn_paged.cu.
#include <cuda_bf16.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "attn_common.cuh"
#include "attn_paged.cuh"
#include "tcgen05.cuh"

namespace ris {

// Device error word of this file (bit 1: a token or key outside the pages); read by ris_device_status.
__device__ unsigned int g_ris_paged_error;

namespace {

using namespace paged;

// ---------------------------------------------------------------- writing rows
// Threads take 16-byte pieces of a CTA's rows of k and v, all of a thread's loads before its stores. Bound by
// HBM, each row read and written once; a row's place is a chain of loads (sequence, start, page), which is
// all that a call of few rows takes.
constexpr int kAppendThreads = 128, kAppendPieces = 2, kAppendOne = 1024;  // (pieces that one CTA takes alone, in several steps)

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
        // (step by step for all pieces, without a branch in between: 32,100 rows of 2 heads of 128 take 12.1 us, 80% of the copy
        // rate; four pieces to a thread, one chain after another, took 13.7)
        uint4 k[U], v[U];
        int64_t at[U], slot[U];
        int seq[U], e[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int t = min(t0 + u * kAppendThreads, n - 1);
            const int64_t row = r0 + t / pieces;
            e[u] = t % pieces * V;
            seq[u] = a.seq_of[row];
            k[u] = *reinterpret_cast<const uint4 *>(reinterpret_cast<const T *>(a.k) + row * a.k_stride + e[u]);
            v[u] = *reinterpret_cast<const uint4 *>(reinterpret_cast<const T *>(a.v) + row * a.v_stride + e[u]);
            slot[u] = row;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) slot[u] += (int64_t)start[seq[u]] - a.off[seq[u]];
        bool lost = false;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool in = slot[u] >= 0 && slot[u] >> a.c.page_log2 < a.c.table_len;
            const int page = page_of(a.c, seq[u], in ? (int)slot[u] : 0), d = e[u] / a.c.D;
            at[u] = in && page >= 0 ? slot_at(a.c, page, d, (int)slot[u]) + e[u] - d * a.c.D : -1;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (t0 + u * kAppendThreads >= n) continue;
            lost = lost || at[u] < 0;
            if (at[u] < 0) continue;
            *reinterpret_cast<uint4 *>(reinterpret_cast<T *>(a.c.k) + at[u]) = k[u];
            *reinterpret_cast<uint4 *>(reinterpret_cast<T *>(a.c.v) + at[u]) = v[u];
        }
        if (lost) atomicOr(&g_ris_paged_error, 1u);
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
    __shared__ int near[kPlanThreads];  // seq_items where they fit
    after_last();
    int *const first = a.c.B <= kPlanThreads ? near : a.seq_items;
    int64_t all, before = 0;
    for (int s0 = 0; s0 < a.c.B; s0 += kPlanThreads) {
        const int s = s0 + threadIdx.x;
        const int tiles = s < a.c.B ? (a.off[s + 1] - a.off[s] + a.tokens - 1) / a.tokens : 0;
        const int64_t at = before + block_scan<kPlanThreads>(tiles, mem, all);
        if (s < a.c.B) first[s] = (int)at;
        before += all;
    }
    const int n = (int)before;
    __syncthreads();  // (they are read by the whole block)
    before = 0;
    for (int i0 = 0; i0 < n; i0 += kPlanThreads) {
        const int i = i0 + threadIdx.x;
        int64_t cost = 0;
        if (i < n) {
            int lo = 0, hi = a.c.B - 1;  // the last sequence whose first item is at or before i
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (first[mid] <= i)
                    lo = mid;
                else
                    hi = mid - 1;
            }
            const PagedItem it{lo, i - first[lo]};
            a.items[i] = it;
            cost = sight_of<KEYS>(a, length_of(a, lo), a.off[lo + 1] - a.off[lo], it.tile).n + a.unit_cost;
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
        constexpr int AT_ONCE = 4;  // (their loads all at once: a call of few rows is a chain of latencies)
        for (int c0 = sp.first + wr; c0 <= sp.last; c0 += AT_ONCE * W) {
            float4 y[AT_ONCE];
            float z[AT_ONCE][C];
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                const int c = min(c0 + i * W, sp.last);
                y[i] = a.part_ml[place(c)];
                if (c0 + i * W > sp.last) y[i].y = 0.f;
                const float *p = a.part_o + place(c) * D + C * lane;
                if constexpr (C == 4) {
                    const float4 q = *reinterpret_cast<const float4 *>(p);
                    z[i][0] = q.x, z[i][1] = q.y, z[i][2] = q.z, z[i][3] = q.w;
                } else {
                    const float2 q = *reinterpret_cast<const float2 *>(p);
                    z[i][0] = q.x, z[i][1] = q.y;
                }
            }
            // (a part without a visible key adds nothing, whatever its product holds)
            float top = m;
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) top = y[i].y == 0.f ? top : fmaxf(top, y[i].x);
            const float ref = top == -INFINITY ? 0.f : top, al = exp2f(m - ref);
            m = top;
            l *= al, n *= al;
#pragma unroll
            for (int e = 0; e < C; ++e) o[e] *= al;
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                if (y[i].y == 0.f) continue;
                const float f = exp2f(y[i].x - ref);
                l = fmaf(y[i].y, f, l);
                n = fmaf(y[i].z, f, n);
#pragma unroll
                for (int e = 0; e < C; ++e) o[e] = fmaf(z[i][e], f, o[e]);
            }
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
// A CTA walks its run of tiles of 8 R rows and 64 keys with a running maximum and sum. Keys and values come row by
// row by cp.async into a buffer each, the next keys under the value product and the next values under the
// scores; two CTAs of an SM fill each other's phases. S: a patch of R x 4 per thread, 4 elements at a time as packed
// pairs; the softmax over the 16 lanes that share a row; O += P V with a patch of R x D / 16. Rows of Q, K and P lie in
// 16-byte pieces swizzled by the row's low three bits, so that the rows that a warp reads at once lie in different banks.
// 4 D flops per row and key on the FMA pipe, which runs at 45% of its rate in long chunks (35 TFLOP/s; 900 tokens behind
// 301 at 12 / 2 heads of 128: 156 us): the rest goes to operands. A patch of 4 x 4 in tiles of 32 rows took 208 us, 4 x 4
// with twice the threads on 64 rows 167. Tiles of 8 rows (R = 1) are for single tokens: 16 of them behind 8,000 keys
// take 124 us (2.1 TB/s) instead of 150 in tiles of 32.
constexpr int BN = kPagedF32Keys;
constexpr int kF32Threads = 128, TY = kF32Threads / 16;  // (rows ty + TY i, keys tx + 16 j)
static_assert(TY == 8 && BN == 64, "the swizzle; a thread's four keys");

using tc::f2_fma;
using tc::f2_mul;
using tc::f2_pack;
using tc::f2_unpack;

__device__ __forceinline__ void store4(float *p, float4 x) { *reinterpret_cast<float4 *>(p) = x; }
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

// The keys (or values) of a tile that some row of the unit sees, the others as zeros
template <int D, bool SWIZZLE>
__device__ __forceinline__ void fetch_keys(const PagedAttendArgs &a, const Unit &u, float *dst, const void *pool, int k0)
{
    constexpr int AT_ONCE = kF32Threads / (D / 4);  // rows
    const int w = threadIdx.x / (D / 4), d = threadIdx.x % (D / 4);
#pragma unroll 2
    for (int r0 = 0; r0 < BN; r0 += 16) {  // (16 keys of a tile lie in one page)
        const int j0 = k0 + r0;
        const bool wanted = j0 < u.sight.end && (j0 + 15 >= u.sight.low || j0 < a.anchors);
        const int page = wanted ? page_of(a.c, u.seq, j0) : -1;
        if (wanted && page < 0) atomicOr(&g_ris_paged_error, 1u);
        const float *src = reinterpret_cast<const float *>(pool) + (page >= 0 ? slot_at(a.c, page, u.kv_head, j0 + w) + 4 * d : 0);
        const int64_t step = page >= 0 ? AT_ONCE * a.c.slot_stride : 0;
#pragma unroll
        for (int e = 0; e < 16 / AT_ONCE; ++e, src += step) {
            const int r = r0 + e * AT_ONCE + w, j = k0 + r;
            copy16(dst + r * D + 4 * (SWIZZLE ? d ^ (r & 7) : d), src, page >= 0 && j < u.sight.end && (j >= u.sight.low || j < a.anchors));
        }
    }
    copies_end();
}

template <int D, int R>
__global__ void __launch_bounds__(kF32Threads, 2) k_paged_f32(const __grid_constant__ PagedAttendArgs a)
{
    constexpr int BM = TY * R, C = D / 16;  // columns of O of a thread
    extern __shared__ __align__(16) float sm[];
    float *const qs = sm, *const ks = qs + BM * D, *const vs = ks + BN * D, *const ps = vs + BN * D;
    __shared__ RunMem mem;
    after_last();
    const Run run = run_of<BN, kF32Threads>(a, blockIdx.x, mem);
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;  // rows ty + TY i; keys tx + 16 j; columns 4 tx + 64 c
    PagedSplit split{-1};
    Walk walk(run);
    Unit u;
    while (walk.next<BN>(a, run, u)) {
        if (u.split.first >= 0) split = u.split;
        __syncthreads();  // the last unit's buffers are free
        // the query rows: token r / block, head r % block; zeros for rows that there are not
        for (int t = threadIdx.x; t < BM * (D / 4) && u.j0 < u.j1; t += kF32Threads) {
            const int r = t / (D / 4), d = t % (D / 4), tok = r / a.block, h = r % a.block;
            const bool there = tok < u.sight.tokens && h < u.heads;
            const float *q = reinterpret_cast<const float *>(a.q) + (there ? (int64_t)(u.row0 + tok) * a.q_stride + (u.head0 + h) * D + 4 * d : 0);
            copy16(qs + r * D + 4 * (d ^ (r & 7)), q, there);
        }
        if (u.j0 < u.j1) {
            fetch_keys<D, true>(a, u, ks, a.c.k, BN * u.sight.granule(u.j0));
            fetch_keys<D, false>(a, u, vs, a.c.v, BN * u.sight.granule(u.j0));
        }
        int pos[R];  // of each row; one that is not there sees nothing
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int r = ty + TY * i, tok = r / a.block;
            pos[i] = tok < u.sight.tokens && r % a.block < u.heads ? u.sight.pos0 + tok : -1;
        }
        uint64_t o[R][C / 2] = {};
        float m[R], l[R];
#pragma unroll
        for (int i = 0; i < R; ++i) m[i] = -INFINITY, l[i] = 0.f;
        for (int t = u.j0; t < u.j1; ++t) {
            const int k0 = BN * u.sight.granule(t);
            const bool more = t + 1 < u.j1;
            // whether every row sees the whole tile
            const bool whole = k0 + BN - 1 <= u.sight.pos0 && (k0 + BN <= a.anchors || a.window == 0 || u.sight.pos0 + u.sight.tokens - 1 - k0 < a.window);
            copied_but<1>();  // (the values' copy may still be on its way)
            __syncthreads();
            uint64_t s2[R][4] = {};  // two partial sums of each score: of the even and of the odd elements
#pragma unroll 2
            for (int d = 0; d < D / 4; ++d) {
                ulonglong2 kb[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) kb[j] = *reinterpret_cast<const ulonglong2 *>(ks + (tx + 16 * j) * D + 4 * (d ^ (tx & 7)));
#pragma unroll
                for (int i = 0; i < R; ++i) {
                    const ulonglong2 qa = *reinterpret_cast<const ulonglong2 *>(qs + (ty + TY * i) * D + 4 * (d ^ ty));
#pragma unroll
                    for (int j = 0; j < 4; ++j) s2[i][j] = f2_fma(qa.x, kb[j].x, s2[i][j]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) s2[i][j] = f2_fma(qa.y, kb[j].y, s2[i][j]);
                }
            }
            __syncthreads();  // the keys' buffer is free
            if (more)
                fetch_keys<D, true>(a, u, ks, a.c.k, BN * u.sight.granule(t + 1));
            else
                copies_end();
#pragma unroll
            for (int i = 0; i < R; ++i) {
                float s[4], mx = -INFINITY;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float x, y;
                    f2_unpack(s2[i][j], x, y);
                    s[j] = (x + y) * a.scale_log2;
                    if (!whole && !sees(a, pos[i], k0 + tx + 16 * j)) s[j] = -INFINITY;
                    mx = fmaxf(mx, s[j]);
                }
#pragma unroll
                for (int x = 8; x > 0; x >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, x));
                const float nm = fmaxf(m[i], mx), ref = nm == -INFINITY ? 0.f : nm;
                const float al = exp2f(m[i] - ref);
                m[i] = nm;
                float sum = 0.f;
                float *const p = ps + (ty + TY * i) * BN + (tx & 3);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    s[j] = exp2f(s[j] - ref);
                    sum += s[j];
                    p[4 * ((tx / 4 + 4 * j) ^ ty)] = s[j];
                }
                l[i] = fmaf(l[i], al, sum);  // this lane's part of the row's sum
                const uint64_t al2 = f2_pack(al, al);
#pragma unroll
                for (int c = 0; c < C / 2; ++c) o[i][c] = f2_mul(o[i][c], al2);
            }
            copied_but<1>();  // (the next keys' copy may still be on its way)
            __syncthreads();
            // O += P V; where some row does not see the whole tile, a row takes only the keys that it sees (0 times
            // an infinity or NaN in a key's place is not 0)
            auto values = [&](auto masked) {
#pragma unroll 2
                for (int j = 0; j < BN; j += 4) {
                    float4 p4[R];
#pragma unroll
                    for (int i = 0; i < R; ++i) p4[i] = *reinterpret_cast<const float4 *>(ps + (ty + TY * i) * BN + 4 * ((j / 4) ^ ty));
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        ulonglong2 vb[C / 4];
#pragma unroll
                        for (int c = 0; c < C / 4; ++c) vb[c] = *reinterpret_cast<const ulonglong2 *>(vs + (j + e) * D + 64 * c + 4 * tx);
#pragma unroll
                        for (int i = 0; i < R; ++i) {
                            if (decltype(masked)::value && !sees(a, pos[i], k0 + j + e)) continue;
                            const float p = e == 0 ? p4[i].x : e == 1 ? p4[i].y : e == 2 ? p4[i].z : p4[i].w;
                            const uint64_t pp = f2_pack(p, p);
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
                fetch_keys<D, false>(a, u, vs, a.c.v, BN * u.sight.granule(t + 1));
            else
                copies_end();
        }
        copied_but<0>();
#pragma unroll
        for (int i = 0; i < R; ++i) {
            float sum = l[i];
#pragma unroll
            for (int x = 8; x > 0; x >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, x);
            const int r = ty + TY * i, tok = r / a.block, h = r % a.block;
            if (tok >= u.sight.tokens || h >= u.heads) continue;
            const int64_t row = u.row0 + tok;
            const float inv = u.part >= 0 ? 1.f : sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;  // no key: zeros; NaN stays
            float *to;
            if (u.part < 0) {
                to = reinterpret_cast<float *>(a.out) + (row * a.Hq + u.head0 + h) * D;
                if (tx == 0 && a.lse != nullptr) a.lse[(u.head0 + h) * a.q_total + row] = (m[i] + log2f(sum)) * kLn2;
            } else {
                const int64_t at = (int64_t)u.part * a.part_rows + r;
                to = a.part_o + at * D;
                if (tx == 0) a.part_ml[at] = make_float4(m[i], sum, sum, 0.f);
            }
#pragma unroll
            for (int c = 0; c < C / 4; ++c) {
                float4 y;
                f2_unpack(o[i][2 * c], y.x, y.y);
                f2_unpack(o[i][2 * c + 1], y.z, y.w);
                store4(to + 64 * c + 4 * tx, make_float4(y.x * inv, y.y * inv, y.z * inv, y.w * inv));
            }
        }
    }
    if (threadIdx.x == 0) a.split[blockIdx.x] = split;
}

template <int D, int R>
cudaError_t launch_f32(const PagedAttendArgs &a, cudaStream_t s)
{
    constexpr int bytes = ((TY * R + 2 * BN) * D + TY * R * BN) * (int)sizeof(float);
    static_assert(2 * (bytes + (int)sizeof(RunMem) + 1024) <= 228 * 1024, "two CTAs of an SM");
    static Once once;
    const cudaError_t ready = once([] { return cudaFuncSetAttribute(k_paged_f32<D, R>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes); });
    if (ready != cudaSuccess) return ready;
    return launch_chained(k_paged_f32<D, R>, dim3((unsigned)a.runs), dim3(kF32Threads), bytes, s, a);
}

template <typename T, int D>
cudaError_t launch_join(const PagedAttendArgs &a, cudaStream_t s)
{
    // few rows of many parts (8 or more to a row tile): every warp of a CTA on the parts of one row, else a row for each (48
    // row tiles of 24 rows and about 4 parts: 8.4 us instead of 5.1)
    if (a.part_rows <= 32 && a.runs >= 8 * a.line) return launch_chained(k_paged_join<T, D, kJoinWarps>, dim3((unsigned)a.runs, (unsigned)a.part_rows), dim3(kJoinThreads), 0, s, a);
    return launch_chained(k_paged_join<T, D, 1>, dim3((unsigned)a.runs, (unsigned)((a.part_rows + kJoinWarps - 1) / kJoinWarps)), dim3(kJoinThreads), 0, s, a);
}

}  // namespace

cudaError_t launch_paged_append(PagedAppendArgs a, int dtype, cudaStream_t s)
{
    const int pieces = a.c.Hkv * a.c.D / (dtype == RIS_F32 ? 4 : 8);
    constexpr int64_t full = kAppendThreads * kAppendPieces;  // of a CTA
    // one CTA where it can take everything, else full ones, or two on every SM
    const int64_t most = std::max<int64_t>(1, full / pieces);
    a.rows = (int)(a.total * pieces <= kAppendOne ? a.total : std::min<int64_t>(most, std::max<int64_t>(1, a.total / (2 * kPagedSMs))));
    int64_t blocks = 0;
    if (a.total > 0) {
        blocks = (a.total + a.rows - 1) / a.rows;
        const cudaError_t e = dtype == RIS_F32 ? launch_chained(k_paged_append<float>, dim3((unsigned)blocks), dim3(kAppendThreads), 0, s, a)
                                               : launch_chained(k_paged_append<__nv_bfloat16>, dim3((unsigned)blocks), dim3(kAppendThreads), 0, s, a);
        if (e != cudaSuccess) return e;
    }
    if (blocks == 1 || (blocks > 0 && a.start != nullptr)) return cudaSuccess;
    // (without rows too: lengths outside the slots are cut)
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

// Rows of a row tile: the smallest that takes the most that a sequence has of them.
int32_t paged_f32_rows(int64_t rows) { return rows <= 8 ? 8 : rows <= 32 ? 32 : 64; }

cudaError_t launch_paged_f32(const PagedAttendArgs &a, int32_t rows, cudaStream_t s)
{
    if (rows == 8) return a.c.D == 128 ? launch_f32<128, 1>(a, s) : launch_f32<64, 1>(a, s);
    if (rows == 32) return a.c.D == 128 ? launch_f32<128, 4>(a, s) : launch_f32<64, 4>(a, s);
    return a.c.D == 128 ? launch_f32<128, 8>(a, s) : launch_f32<64, 8>(a, s);
}

cudaError_t paged_error_word(unsigned int **p) { return cudaGetSymbolAddress(reinterpret_cast<void **>(p), g_ris_paged_error); }

}  // namespace ris
