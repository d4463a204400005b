// Cutting a cache back to a budget by accumulated attention weight.
//
// Of the slots of a (sequence, KV head) the `budget` first in this order stay: those of the newest
// positions (within `recent` of the newest one), then by weight, then by slot. The keys are rotated and carry their
// positions, so slots need no order: a kept slot below the budget stays where it is, and the i-th
// kept one above it moves into the i-th freed one, which moves no more rows than have to move and
// lets every row move at once, in place too (all sources lie at or above the budget, all targets
// below it).
#include <cstdint>

#include "serve.h"

namespace ris {
namespace {

// The weight's place in the order as an unsigned number: larger is heavier; -0 as 0, NaN lightest.
__device__ __forceinline__ uint32_t order_of(float w)
{
    const uint32_t u = __float_as_uint(w + 0.f);
    if ((u & 0x7FFFFFFFu) > 0x7F800000u) return 0u;
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

constexpr int kThreads = 1024, kWarps = kThreads / 32;

// Sum over the block of x, and this thread's exclusive prefix.
__device__ __forceinline__ int block_scan(int x, int &total)
{
    __shared__ int part[kWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int inc = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xFFFFFFFFu, inc, o);
        if (lane >= o) inc += y;
    }
    __syncthreads();
    if (lane == 31) part[warp] = inc;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        before += w < warp ? part[w] : 0;
        all += part[w];
    }
    total = all;
    return before + inc - x;
}

// One CTA per (sequence, KV head): the newest position, the threshold weight by four passes over
// eight bits each, then the lists in slot order. holes: [B * Hkv][budget] scratch.
__global__ void __launch_bounds__(kThreads) k_evict_select(const Cache4EvictArgs a, int32_t *holes)
{
    __shared__ int hist[256];
    __shared__ int sh_max, sh_digit, sh_need;
    const int bh = blockIdx.x, b = bh / a.src.Hkv, tid = threadIdx.x;
    const int len = max(0, (int)min((int64_t)a.src.length[b], a.src.cap));
    const int left = min(len, a.budget);
    const float *weight = a.src.weight + bh * a.src.cap;
    const int32_t *pos = a.src.pos + bh * a.src.cap;
    int32_t *kept = a.kept + (int64_t)bh * a.budget;
    holes += (int64_t)bh * a.budget;
    if (len <= a.budget) {
        for (int j = tid; j < a.budget; j += kThreads) kept[j] = j < len ? j : -1;
        return;
    }
    if (tid == 0) sh_max = INT32_MIN;
    __syncthreads();
    int newest = INT32_MIN;
    for (int j = tid; j < len; j += kThreads) newest = max(newest, pos[j]);
    atomicMax(&sh_max, newest);
    __syncthreads();
    const int64_t line = (int64_t)sh_max - a.recent;  // newer than this: recent
    int mine = 0, n_recent;
    for (int j = tid; j < len; j += kThreads) mine += pos[j] > line;
    block_scan(mine, n_recent);
    // the threshold lies among the recent slots (all of the budget goes to them) or among the others
    const bool among_recent = n_recent >= a.budget;
    int need = among_recent ? a.budget : a.budget - n_recent;  // slots to take of that class
    uint32_t prefix = 0, mask = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (tid < 256) hist[tid] = 0;
        __syncthreads();
        for (int j = tid; j < len; j += kThreads) {
            if ((pos[j] > line) != among_recent) continue;
            const uint32_t u = order_of(weight[j]);
            if ((u & mask) == prefix) atomicAdd(&hist[(u >> shift) & 255], 1);
        }
        __syncthreads();
        if (tid == 0) {
            int d = 255, n = need;
            while (d > 0 && hist[d] < n) n -= hist[d--];
            sh_digit = d;
            sh_need = n;
        }
        __syncthreads();
        prefix |= (uint32_t)sh_digit << shift;
        mask |= 255u << shift;
        need = sh_need;
        __syncthreads();
    }
    // slots above the threshold stay, and of those at it the first `need`
    int ties = 0, n_holes = 0, n_moved = 0;
    for (int j0 = 0; j0 < len; j0 += kThreads) {
        const int j = j0 + tid;
        bool keep = false, tie = false;
        if (j < len) {
            const bool rec = pos[j] > line;
            const uint32_t u = order_of(weight[j]);
            if (rec != among_recent)
                keep = rec;
            else {
                keep = u > prefix;
                tie = u == prefix;
            }
        }
        int n;
        const int before = block_scan(tie, n);
        if (tie && ties + before < need) keep = true;
        ties += n;
        const bool hole = j < left && !keep;
        const int h = block_scan(hole, n);
        if (hole) holes[n_holes + h] = j;
        if (j < left && keep) kept[j] = j;
        n_holes += n;
        // movers are met after every slot below the budget, so after every hole (which the scans'
        // barriers order within the block)
        const bool moved = j < len && j >= left && keep;
        const int r = block_scan(moved, n);
        if (moved) kept[holes[n_moved + r]] = j;
        n_moved += n;
    }
}

// Moves the rows: 16 lanes to a slot of the target. Codes 16 bytes at a time; scales, position and weight by single
// lanes. In place only what moves.
constexpr int kMoveThreads = 256;
template <int D>
__global__ void __launch_bounds__(kMoveThreads) k_evict_move(const Cache4EvictArgs a)
{
    constexpr int P = D / 32, LANES = 16;  // 16-byte pieces of a row's codes
    const int64_t t = (int64_t)blockIdx.x * (kMoveThreads / LANES) + threadIdx.x / LANES;
    const int u = threadIdx.x % LANES;
    const int64_t n = (int64_t)a.src.B * a.src.Hkv * a.budget;
    if (t < n) {
        const int64_t bh = t / a.budget, j = t - bh * a.budget;
        const int from = a.kept[t];
        if (from >= 0 && !(a.in_place && from == j)) {
            const int64_t rs = bh * a.src.cap + from, rd = bh * a.dst.cap + j;
            if (u < P)
                reinterpret_cast<uint4 *>(a.dst.k)[rd * P + u] = reinterpret_cast<const uint4 *>(a.src.k)[rs * P + u];
            else if (u < 2 * P)
                reinterpret_cast<uint4 *>(a.dst.v)[rd * P + u - P] = reinterpret_cast<const uint4 *>(a.src.v)[rs * P + u - P];
            else if (u < 2 * P + P / 2)
                reinterpret_cast<uint32_t *>(a.dst.k_scale)[rd * (P / 2) + u - 2 * P] =
                    reinterpret_cast<const uint32_t *>(a.src.k_scale)[rs * (P / 2) + u - 2 * P];
            else if (u < 3 * P)
                reinterpret_cast<uint32_t *>(a.dst.v_scale)[rd * (P / 2) + u - 2 * P - P / 2] =
                    reinterpret_cast<const uint32_t *>(a.src.v_scale)[rs * (P / 2) + u - 2 * P - P / 2];
            else if (u == 3 * P)
                a.dst.pos[rd] = a.src.pos[rs];
            else if (u == 3 * P + 1)
                a.dst.weight[rd] = a.src.weight[rs];
        }
    }
    if (blockIdx.x == 0)
        for (int b = threadIdx.x; b < a.src.B; b += kMoveThreads)
            a.dst.length[b] = max(0, min((int)min((int64_t)a.src.length[b], a.src.cap), a.budget));
}

}  // namespace

cudaError_t launch_cache4_evict(const Cache4EvictArgs &a, int32_t *holes, cudaStream_t s)
{
    k_evict_select<<<(unsigned)(a.src.B * a.src.Hkv), kThreads, 0, s>>>(a, holes);
    cudaError_t e = cudaGetLastError();
    note_launch();
    if (e != cudaSuccess) return e;
    const int64_t n = (int64_t)a.src.B * a.src.Hkv * a.budget, per = kMoveThreads / 16;
    if (a.src.D == 128)
        k_evict_move<128><<<(unsigned)((n + per - 1) / per), kMoveThreads, 0, s>>>(a);
    else
        k_evict_move<64><<<(unsigned)((n + per - 1) / per), kMoveThreads, 0, s>>>(a);
    note_launch();
    return cudaGetLastError();
}

}  // namespace ris
