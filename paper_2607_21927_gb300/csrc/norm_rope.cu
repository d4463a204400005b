// Queries and keys normed per head and turned to their positions in one pass, and the gradient of that.
//
// With h = r x, r = (mean_c x_c^2 + eps)^-1/2 over a head's channels, and z = w h (without a weight z = x):
//   y = m R z on the first `rot` channels, R turning the pair (z_a, z_b) of frequency f by a = f pos, y = z
//   on the others; the pairs are (c, c + rot / 2), or neighbours (2c, 2c + 1).
// Backwards, with g = m R^T dy (g = dy on the channels that are not turned) and u = w g:
//   dx = r (u - h mean_c(u h)),   dw_c = sum over tokens and heads of g_c h_c.
//
// V = 16 / sizeof(T); a thread holds V pairs of a head, both channels of each, as two 16-byte pieces, so that
// the turn needs no other lane: D / 2V lanes make a head, and its sums take log2 of that many exchanges. A
// thread keeps its V angles for all heads of its token. Arithmetic and statistics are fp32 (two values to an
// instruction), angles 64-bit fractions of a turn (rows.cuh). Bound by HBM, each element read once and written
// once: 30,011 tokens of 12 / 2 heads of 128 in bf16 take 38 us (215 MB, 83% of the copy rate); the gradient
// at 32 / 4 heads of 64 takes 69.5 us (415 MB, 88%; 4 more without the hint that the next 256 bytes follow).
#include <algorithm>
#include <cstdint>

#include "rows.cuh"
#include "serve.h"
#include "tcgen05.cuh"

namespace ris {
namespace {

using rows::sincos_half_turns;
using rows::Vec;
using tc::f2_fma;
using tc::f2_mul;
using tc::f2_pack;
using tc::f2_unpack;

constexpr int kThreads = 256, kSMs = 152;
// CTAs of an SM and stages of the ring. Four CTAs (64 registers) took 41 us instead of 37 forwards, three (84) 111 instead
// of 77 backwards; rings of 3 or 6 stages instead of 4 1 us more, of 4 instead of 3 2 us.
constexpr int kForwardCtas = 3, kForwardStages = 4, kBackwardCtas = 2, kBackwardStages = 3;

// The pairs of a thread: lane l of a head's D / 2V.
template <typename T, bool PAIRS, int D>
struct Lane {
    static constexpr int V = Vec<T>::V;
    int at[2];      // first channel of its two pieces; lanes' pieces lie side by side: a sector asked for twice, half each time, took 113 us instead of 77
    int f[2];       // first frequency of its first and of its second V / 2 pairs
    bool turns[2];  // whether these are among the first `rot` channels
    __device__ __forceinline__ Lane(int l, int rot)
    {
        if constexpr (PAIRS) {  // a piece holds V / 2 pairs
            for (int i = 0; i < 2; ++i) {
                at[i] = V * l + i * (D / 2);
                f[i] = at[i] / 2;
                turns[i] = at[i] < rot;
            }
        } else {
            const int n = rot / (2 * V);  // lanes that turn
            turns[0] = turns[1] = l < n;
            at[0] = l < n ? V * l : rot + V * (l - n);
            at[1] = at[0] + (l < n ? rot : D - rot) / 2;
            f[0] = V * l, f[1] = f[0] + V / 2;
        }
    }
    __device__ __forceinline__ bool any() const { return turns[0] || turns[1]; }
    // channels 2 j and 2 j + 1 of the thread's first V (i = 0) or of its second (i = 1), as fp32
    static __device__ __forceinline__ uint64_t get(const Vec<T> (&p)[2], int i, int j)
    {
        if constexpr (PAIRS) return f2_pack(p[(4 * j + i) / V][(4 * j + i) % V], p[(4 * j + 2 + i) / V][(4 * j + 2 + i) % V]);
        return f2_pack(p[i][2 * j], p[i][2 * j + 1]);
    }
    static __device__ __forceinline__ void put(T *row, const int (&at)[2], const uint64_t (&a)[V / 2], const uint64_t (&b)[V / 2])
    {
        float p[2][V];
#pragma unroll
        for (int j = 0; j < V / 2; ++j) {
            float a0, a1, b0, b1;
            f2_unpack(a[j], a0, a1);
            f2_unpack(b[j], b0, b1);
            if constexpr (PAIRS) {
                float *const q = p[4 * j / V] + 4 * j % V;
                q[0] = a0, q[1] = b0, q[2] = a1, q[3] = b1;
            } else {
                p[0][2 * j] = a0, p[0][2 * j + 1] = a1;
                p[1][2 * j] = b0, p[1][2 * j + 1] = b1;
            }
        }
        Vec<T>::store(row + at[0], p[0]);
        Vec<T>::store(row + at[1], p[1]);
    }
    static __device__ __forceinline__ void load(Vec<T> (&p)[2], const T *row, const int (&at)[2])
    {
        p[0].load(row + at[0]);
        p[1].load(row + at[1]);
    }
};

// x summed over the n lanes of a head (n a power of two, aligned)
__device__ __forceinline__ float head_sum(float x, int n)
{
    for (int o = n >> 1; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
    return x;
}

// The work is a line of steps, a head of TOKENS tokens each, heads innermost; every CTA takes an equal run of it.
struct Steps {
    int64_t first, end;
    __device__ __forceinline__ Steps(int64_t groups, int heads, int64_t cta, int64_t ctas)
    {
        const int64_t all = groups * heads, each = all / ctas, more = all % ctas;
        first = each * cta + min(cta, more);
        end = first + each + (cta < more ? 1 : 0);
    }
};

// Where a thread is on the line: its token's row (row 0 past the last token), the head.
template <int TOKENS>
struct Place {
    int64_t group, row;
    int head;
    bool there;
    __device__ __forceinline__ Place(int64_t step, int heads, int64_t n) : group(step / heads), head((int)(step % heads)) { find(n); }
    __device__ __forceinline__ void find(int64_t n)
    {
        const int64_t p = group * TOKENS + threadIdx.x / (kThreads / TOKENS);
        there = p < n;
        row = there ? p : 0;
    }
    __device__ __forceinline__ bool next(int heads, int64_t n)  // whether it is another group's
    {
        if (++head < heads) return false;
        head = 0;
        ++group;
        find(n);
        return true;
    }
};

// Steps on their way: S stages of P pieces for every thread, each read by the thread that asked for it (no
// barrier), so that what is in flight takes no registers: with the loads in registers, one or two heads ahead, these
// took 46 and 97 us.
template <int S, int P>
struct Ring {
    uint4 *mine;
    __device__ __forceinline__ explicit Ring(uint4 *mem) : mine(mem + threadIdx.x) {}
    __device__ __forceinline__ uint4 *at(int64_t step, int piece) const { return mine + ((int)(step % S) * P + piece) * kThreads; }
    __device__ __forceinline__ void ask(int64_t step, int piece, const void *src) const
    {
        asm volatile("cp.async.cg.shared.global.L2::256B [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(at(step, piece))), "l"(src) : "memory");
    }
    static __device__ __forceinline__ void close() { asm volatile("cp.async.commit_group;" ::: "memory"); }
    static __device__ __forceinline__ void wait() { asm volatile("cp.async.wait_group %0;" ::"n"(S - 2) : "memory"); }  // for the oldest of S - 1
    static constexpr int BYTES = S * P * kThreads * 16;
};

// cos and sin, times mscale, of a thread's V frequencies; its channels turned on by them, or back
template <int V>
struct Turn {
    uint64_t cs[V / 2], sn[V / 2];
    template <typename L>
    __device__ __forceinline__ void at(const NormRopeArgs &a, const L &lane, int32_t pos)
    {
#pragma unroll
        for (int j = 0; j < V / 2; ++j) {
            if (!lane.turns[4 * j / V]) continue;
            const uint64_t *const f = a.turn + lane.f[4 * j / V] + 2 * j % (V / 2);
            float s0, s1, c0, c1;
            sincos_half_turns(pos, f[0], &s0, &c0);
            sincos_half_turns(pos, f[1], &s1, &c1);
            cs[j] = f2_pack(c0 * a.mscale, c1 * a.mscale);
            sn[j] = f2_pack(s0 * a.mscale, s1 * a.mscale);
        }
    }
    template <bool BACK, typename L>
    __device__ __forceinline__ void turn(const L &lane, uint64_t (&u)[V / 2], uint64_t (&v)[V / 2]) const
    {
        constexpr uint64_t minus = 0x8000000080000000ull;
#pragma unroll
        for (int j = 0; j < V / 2; ++j) {
            if (!lane.turns[4 * j / V]) continue;
            const uint64_t x = u[j], y = v[j];
            u[j] = f2_fma(x, cs[j], f2_mul(y, BACK ? sn[j] : sn[j] ^ minus));
            v[j] = f2_fma(y, cs[j], f2_mul(x, BACK ? sn[j] ^ minus : sn[j]));
        }
    }
};

// the thread's part of a tensor's weight, ones without
template <typename L, int V, typename T>
__device__ __forceinline__ void load_weight(const T *w, const int (&at)[2], uint64_t (&wa)[V / 2], uint64_t (&wb)[V / 2])
{
    Vec<T> p[2];
    if (w != nullptr) L::load(p, w, at);
#pragma unroll
    for (int j = 0; j < V / 2; ++j) {
        wa[j] = w != nullptr ? L::get(p, 0, j) : f2_pack(1.f, 1.f);
        wb[j] = w != nullptr ? L::get(p, 1, j) : f2_pack(1.f, 1.f);
    }
}
__device__ __forceinline__ float both(uint64_t x)
{
    float a, b;
    f2_unpack(x, a, b);
    return a + b;
}

template <typename T, bool PAIRS, int D>
__global__ void __launch_bounds__(kThreads, kForwardCtas) k_norm_rope(const __grid_constant__ NormRopeArgs a)
{
    using L = Lane<T, PAIRS, D>;
    using R = Ring<kForwardStages, 2>;
    constexpr int V = L::V, LANES = D / (2 * V), TOKENS = kThreads / LANES;
    extern __shared__ __align__(16) uint4 mem[];
    const L lane(threadIdx.x % LANES, a.rot);
    const R ring(mem);
    after_last();
    const int heads = a.heads[0] + a.heads[1];  // of q, then of k
    const Steps run((a.n + TOKENS - 1) / TOKENS, heads, blockIdx.x, gridDim.x);
    Place<TOKENS> ahead(run.first, heads, a.n), here = ahead;
    int64_t asked = run.first;
    auto ask = [&] {
        if (asked < run.end) {
            const int w = ahead.head >= a.heads[0];
            const T *x = reinterpret_cast<const T *>(a.x[w]) + ahead.row * a.x_stride[w] + (ahead.head - w * a.heads[0]) * D;
            ring.ask(asked, 0, x + lane.at[0]);
            ring.ask(asked, 1, x + lane.at[1]);
            ++asked;
            ahead.next(heads, a.n);
        }
        R::close();
    };
#pragma unroll
    for (int i = 0; i < kForwardStages - 1; ++i) ask();
    Turn<V> turn;
    uint64_t wa[V / 2], wb[V / 2];
    const T *weight = nullptr;
    bool moved = lane.any();
    int of = -1;  // whose weight it is
    for (int64_t s = run.first; s < run.end; ++s) {
        if (moved) turn.at(a, lane, a.pos[here.row]);
        const int w = here.head >= a.heads[0];
        if (w != of) {
            of = w;
            weight = reinterpret_cast<const T *>(a.weight[w]);
            load_weight<L, V>(weight, lane.at, wa, wb);
        }
        R::wait();
        Vec<T> x[2];
        x[0].raw = *ring.at(s, 0);
        x[1].raw = *ring.at(s, 1);
        ask();  // (into the place of the step before)
        uint64_t u[V / 2], v[V / 2];
#pragma unroll
        for (int j = 0; j < V / 2; ++j) u[j] = L::get(x, 0, j), v[j] = L::get(x, 1, j);
        if (weight != nullptr) {  // (the same for all threads)
            uint64_t q = 0;
#pragma unroll
            for (int j = 0; j < V / 2; ++j) q = f2_fma(u[j], u[j], f2_fma(v[j], v[j], q));
            const float r = rsqrtf(fmaf(head_sum(both(q), LANES), 1.f / D, a.eps));
            const uint64_t r2 = f2_pack(r, r);
#pragma unroll
            for (int j = 0; j < V / 2; ++j) {
                u[j] = f2_mul(f2_mul(u[j], r2), wa[j]);
                v[j] = f2_mul(f2_mul(v[j], r2), wb[j]);
            }
        }
        turn.template turn<false>(lane, u, v);
        if (here.there) L::put(reinterpret_cast<T *>(a.y[w]) + here.row * a.y_stride[w] + (here.head - w * a.heads[0]) * D, lane.at, u, v);
        moved = here.next(heads, a.n) && lane.any();
    }
}

// s + c += x, what the addition drops kept in c
__device__ __forceinline__ void add_exactly(float &s, float &c, float x)
{
    const float t = __fadd_rn(s, x), y = __fsub_rn(t, s);
    c = __fadd_rn(c, __fadd_rn(__fsub_rn(s, __fsub_rn(t, y)), __fsub_rn(x, y)));
    s = t;
}

// A thread's sums of a weight's gradient. fp32 additions one after another would be off by up to 2^-24 of the sum each, all the same way where
// the terms are alike (a thousand equal ones: 1e-5): a thread adds up kSumSteps of them in its registers, then these go to pairs of fp32 in its
// column of shared memory, and everything after that is added in pairs.
constexpr int kSumSteps = 64;
template <int V, int LANES>
struct Sums {
    static constexpr int PITCH = kThreads + LANES;  // (the lanes' columns of different channels in different banks)
    static constexpr int BYTES = 2 * V * PITCH * (int)sizeof(float2);
    float2 *mem;
    __device__ __forceinline__ void add(uint64_t (&a)[V / 2], uint64_t (&b)[V / 2], bool first) const
    {
#pragma unroll
        for (int j = 0; j < V / 2; ++j) {
            float x[4];
            f2_unpack(a[j], x[0], x[1]);
            f2_unpack(b[j], x[2], x[3]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float2 *const p = mem + (4 * j + i) * PITCH + threadIdx.x;
                float2 y = first ? make_float2(0.f, 0.f) : *p;
                add_exactly(y.x, y.y, x[i]);
                *p = y;
            }
            a[j] = b[j] = 0;
        }
    }
    // over the block's threads of lane l, in a fixed order
    __device__ __forceinline__ float2 of(int l, int row) const
    {
        float s[4] = {}, c[4] = {};
        for (int g = 0; g < kThreads / LANES; g += 4) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 y = mem[row * PITCH + (g + i) * LANES + l];
                add_exactly(s[i], c[i], y.x);
                c[i] += y.y;
            }
        }
#pragma unroll
        for (int i = 1; i < 4; ++i) {
            add_exactly(s[0], c[0], s[i]);
            c[0] += c[i];
        }
        return make_float2(s[0], c[0]);
    }
};

// The gradient. A CTA belongs to q or to k (the sums of a weight's gradient stay in its threads' registers)
// and takes every step-th group of tokens of it; what its threads summed is added up in a fixed order here
// and over the CTAs in k_weight_sums, so that no result depends on the order in which they run.
template <typename T, bool PAIRS, int D>
__global__ void __launch_bounds__(kThreads, kBackwardCtas) k_norm_rope_backward(const __grid_constant__ NormRopeArgs a)
{
    using L = Lane<T, PAIRS, D>;
    using R = Ring<kBackwardStages, 4>;
    constexpr int V = L::V, LANES = D / (2 * V), TOKENS = kThreads / LANES;
    extern __shared__ __align__(16) uint4 mem[];
    const L lane(threadIdx.x % LANES, a.rot);
    const R ring(mem);
    const Sums<V, LANES> sums{reinterpret_cast<float2 *>(mem + R::BYTES / 16)};
    const int w = (int)blockIdx.x >= a.ctas[0], heads = a.heads[w];
    after_last();
    const T *const weight = reinterpret_cast<const T *>(a.weight[w]);
    const Steps run((a.n + TOKENS - 1) / TOKENS, heads, blockIdx.x - (w ? a.ctas[0] : 0), a.ctas[w]);
    Place<TOKENS> ahead(run.first, heads, a.n), here = ahead;
    int64_t asked = run.first;
    auto ask = [&] {
        if (asked < run.end) {
            const T *d = reinterpret_cast<const T *>(a.dy[w]) + ahead.row * a.dy_stride[w] + ahead.head * D;
            ring.ask(asked, 0, d + lane.at[0]);
            ring.ask(asked, 1, d + lane.at[1]);
            if (weight != nullptr) {
                const T *x = reinterpret_cast<const T *>(a.x[w]) + ahead.row * a.x_stride[w] + ahead.head * D;
                ring.ask(asked, 2, x + lane.at[0]);
                ring.ask(asked, 3, x + lane.at[1]);
            }
            ++asked;
            ahead.next(heads, a.n);
        }
        R::close();
    };
#pragma unroll
    for (int i = 0; i < kBackwardStages - 1; ++i) ask();
    Turn<V> turn;
    uint64_t wa[V / 2], wb[V / 2], ga[V / 2] = {}, gb[V / 2] = {};
    load_weight<L, V>(weight, lane.at, wa, wb);
    bool moved = lane.any();
    for (int64_t s = run.first; s < run.end; ++s) {
        if (moved) turn.at(a, lane, a.pos[here.row]);
        R::wait();
        Vec<T> d[2], x[2];
        d[0].raw = *ring.at(s, 0);
        d[1].raw = *ring.at(s, 1);
        if (weight != nullptr) {
            x[0].raw = *ring.at(s, 2);
            x[1].raw = *ring.at(s, 3);
        }
        ask();  // (into the place of the step before)
        uint64_t ua[V / 2], ub[V / 2];
#pragma unroll
        for (int j = 0; j < V / 2; ++j) ua[j] = L::get(d, 0, j), ub[j] = L::get(d, 1, j);
        turn.template turn<true>(lane, ua, ub);
        if (weight != nullptr) {  // (the same for all threads)
            uint64_t xa[V / 2], xb[V / 2], q = 0, t = 0;
#pragma unroll
            for (int j = 0; j < V / 2; ++j) {
                xa[j] = L::get(x, 0, j), xb[j] = L::get(x, 1, j);
                q = f2_fma(xa[j], xa[j], f2_fma(xb[j], xb[j], q));
                t = f2_fma(f2_mul(ua[j], wa[j]), xa[j], f2_fma(f2_mul(ub[j], wb[j]), xb[j], t));
            }
            const float r = rsqrtf(fmaf(head_sum(both(q), LANES), 1.f / D, a.eps));
            const float mean = head_sum(both(t), LANES) * r * (1.f / D);  // of u h
            const uint64_t r2 = f2_pack(r, r), m2 = f2_pack(-mean, -mean);
#pragma unroll
            for (int j = 0; j < V / 2; ++j) {
                const uint64_t ha = f2_mul(xa[j], r2), hb = f2_mul(xb[j], r2);
                if (here.there) {
                    ga[j] = f2_fma(ua[j], ha, ga[j]);
                    gb[j] = f2_fma(ub[j], hb, gb[j]);
                }
                ua[j] = f2_mul(r2, f2_fma(m2, ha, f2_mul(ua[j], wa[j])));
                ub[j] = f2_mul(r2, f2_fma(m2, hb, f2_mul(ub[j], wb[j])));
            }
        }
        if (here.there) L::put(reinterpret_cast<T *>(a.y[w]) + here.row * a.y_stride[w] + here.head * D, lane.at, ua, ub);
        moved = here.next(heads, a.n) && lane.any();
        if (weight != nullptr && (s - run.first) % kSumSteps == kSumSteps - 1) sums.add(ga, gb, s - run.first == kSumSteps - 1);
    }
    if (weight == nullptr) return;
    sums.add(ga, gb, run.end - run.first < kSumSteps);
    __syncthreads();
    if (threadIdx.x >= D) return;
    // (row of a channel: as Sums::add has them)
    const int row = threadIdx.x / LANES, e = row / 4 * 2 + row % 2, b = row / 2 % 2;
    const L of(threadIdx.x % LANES, a.rot);
    const int p = PAIRS ? 2 * e + b : V * b + e, c = (p < V ? of.at[0] : of.at[1]) + p % V;
    a.part[(int64_t)blockIdx.x * D + c] = sums.of(threadIdx.x % LANES, row);
}

// dw of q (blockIdx.y 0) and k (1), 32 channels to a CTA: the CTAs' sums, a warp on every 32nd of them, then a warp's
// lanes on a channel's. In pairs of fp32: as fp64 additions, of which an SM has few, the same sums took 15 us.
constexpr int kSumWarps = 32;
__global__ void __launch_bounds__(32 * kSumWarps) k_weight_sums(const float2 *part, int D, int ctas_q, int ctas_k, float *gq, float *gk)
{
    __shared__ float2 sums[32][kSumWarps + 1];
    const int w = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n = w ? ctas_k : ctas_q, c0 = 32 * blockIdx.x;
    float *const out = w ? gk : gq;
    after_last();
    if (out == nullptr) return;
    part += (int64_t)(w ? ctas_q : 0) * D + c0 + lane;
    float s = 0.f, c = 0.f;
#pragma unroll 8
    for (int i = warp; i < n; i += kSumWarps) {
        const float2 x = part[(int64_t)i * D];
        add_exactly(s, c, x.x);
        c += x.y;
    }
    sums[lane][warp] = make_float2(s, c);
    __syncthreads();
    const float2 y = sums[warp][lane];
    s = y.x, c = y.y;
    for (int o = 16; o > 0; o >>= 1) {
        const float s2 = __shfl_down_sync(0xFFFFFFFFu, s, o), c2 = __shfl_down_sync(0xFFFFFFFFu, c, o);
        add_exactly(s, c, s2);
        c += c2;
    }
    if (lane == 0) out[c0 + warp] = fabsf(s) < INFINITY ? s + c : s;  // (what an infinity leaves is NaN)
}

template <typename T, bool PAIRS, int D>
cudaError_t forward(const NormRopeArgs &a, cudaStream_t s)
{
    constexpr int TOKENS = kThreads / (D / (2 * Vec<T>::V));
    const int64_t steps = (a.n + TOKENS - 1) / TOKENS * (a.heads[0] + a.heads[1]);
    const unsigned ctas = (unsigned)std::min<int64_t>(steps, kForwardCtas * kSMs);
    return launch_chained(k_norm_rope<T, PAIRS, D>, dim3(ctas), dim3(kThreads), Ring<kForwardStages, 2>::BYTES, s, a);
}

template <typename T, bool PAIRS, int D>
cudaError_t backward(const NormRopeArgs &a, float *gq, float *gk, cudaStream_t s)
{
    if (a.n > 0) {
        constexpr int V = Vec<T>::V, bytes = Ring<kBackwardStages, 4>::BYTES + Sums<V, D / (2 * V)>::BYTES;
        static Once once;
        const cudaError_t ready = once([] { return cudaFuncSetAttribute(k_norm_rope_backward<T, PAIRS, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes); });
        if (ready != cudaSuccess) return ready;
        const cudaError_t e = launch_chained(k_norm_rope_backward<T, PAIRS, D>, dim3((unsigned)(a.ctas[0] + a.ctas[1])), dim3(kThreads), bytes, s, a);
        if (e != cudaSuccess) return e;
    }
    if (gq == nullptr && gk == nullptr) return cudaSuccess;
    const int n0 = a.n > 0 ? a.ctas[0] : 0, n1 = a.n > 0 ? a.ctas[1] : 0;
    return launch_chained(k_weight_sums, dim3(D / 32, 2), dim3(32 * kSumWarps), 0, s, static_cast<const float2 *>(a.part), D, n0, n1, gq, gk);
}

}  // namespace

// CTAs of the gradient's kernel for q and for k: two to an SM in all, shared out by heads, and no more than
// there are steps.
void norm_rope_ctas(int dtype, int D, int64_t n, const int32_t (&heads)[2], int32_t (&ctas)[2])
{
    const int tokens = kThreads / (D / (2 * (dtype == RIS_F32 ? 4 : 8)));
    const int64_t groups = std::max<int64_t>(1, (n + tokens - 1) / tokens);
    const int all = heads[0] + heads[1], most = kBackwardCtas * kSMs;
    ctas[1] = heads[1] == 0 ? 0 : (int32_t)std::min<int64_t>(groups * heads[1], std::max<int64_t>(1, ((int64_t)most * heads[1] + all / 2) / all));
    ctas[0] = (int32_t)std::min<int64_t>(groups * heads[0], std::max(1, most - ctas[1]));
}

cudaError_t launch_norm_rope(const NormRopeArgs &a, int dtype, int D, bool pairs, cudaStream_t s)
{
    if (dtype == RIS_F32) {
        if (D == 128) return pairs ? forward<float, true, 128>(a, s) : forward<float, false, 128>(a, s);
        return pairs ? forward<float, true, 64>(a, s) : forward<float, false, 64>(a, s);
    }
    if (D == 128) return pairs ? forward<__nv_bfloat16, true, 128>(a, s) : forward<__nv_bfloat16, false, 128>(a, s);
    return pairs ? forward<__nv_bfloat16, true, 64>(a, s) : forward<__nv_bfloat16, false, 64>(a, s);
}

cudaError_t launch_norm_rope_backward(const NormRopeArgs &a, int dtype, int D, bool pairs, float *gq, float *gk, cudaStream_t s)
{
    if (dtype == RIS_F32) {
        if (D == 128) return pairs ? backward<float, true, 128>(a, gq, gk, s) : backward<float, false, 128>(a, gq, gk, s);
        return pairs ? backward<float, true, 64>(a, gq, gk, s) : backward<float, false, 64>(a, gq, gk, s);
    }
    if (D == 128) return pairs ? backward<__nv_bfloat16, true, 128>(a, gq, gk, s) : backward<__nv_bfloat16, false, 128>(a, gq, gk, s);
    return pairs ? backward<__nv_bfloat16, true, 64>(a, gq, gk, s) : backward<__nv_bfloat16, false, 64>(a, gq, gk, s);
}

}  // namespace ris
