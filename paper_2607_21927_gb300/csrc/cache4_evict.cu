// Cutting a cache back to a budget by accumulated attention weight.
//
// Of the slots of a (sequence, KV head) the `budget` first in this order stay: those of the newest
// positions (within `recent` of the newest one), then by weight, then by slot. The keys are rotated and
// carry their positions, so slots need no order: a kept slot below the budget stays where it is, and the
// i-th kept one above it moves into the i-th freed one, which moves no more rows than have to move and lets
// every row move at once, in place too (all sources lie at or above the budget, all targets below it).
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

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kBins = 2048, kPasses = 3;  // digits of 11, 11 and 10 bits, from the top
constexpr int kCachedSlots = 20480;       // slots of a CTA whose order and position fit its shared memory

struct Exchange {  // what the CTAs of a cluster read of one another
    int newest, recent, holes, movers;
    uint32_t hist[kPasses][kBins];  // of this CTA's slots
    uint32_t sums[kBins];           // this CTA's share of the cluster's histogram, in its place
};

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// the word at `p` (of this CTA's shared memory) in CTA `rank` of the cluster
__device__ __forceinline__ uint32_t ld_cluster(const void *p, int rank)
{
    uint32_t at, x;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(p)), "r"(rank));
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(x) : "r"(at) : "memory");
    return x;
}

// Sums of (x, y) over the block, and this thread's exclusive prefixes.
struct Pair {
    int x, y;
};
__device__ __forceinline__ Pair block_scan(Pair v, Pair &total, Pair *part)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Pair inc = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int a = __shfl_up_sync(0xFFFFFFFFu, inc.x, o), b = __shfl_up_sync(0xFFFFFFFFu, inc.y, o);
        if (lane >= o) {
            inc.x += a;
            inc.y += b;
        }
    }
    __syncthreads();
    if (lane == 31) part[warp] = inc;
    __syncthreads();
    Pair w = part[lane & (kWarps - 1)];
    if (lane >= kWarps) w = {0, 0};
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int a = __shfl_up_sync(0xFFFFFFFFu, w.x, o), b = __shfl_up_sync(0xFFFFFFFFu, w.y, o);
        if (lane >= o) {
            w.x += a;
            w.y += b;
        }
    }
    total = {__shfl_sync(0xFFFFFFFFu, w.x, 31), __shfl_sync(0xFFFFFFFFu, w.y, 31)};
    const int bx = __shfl_sync(0xFFFFFFFFu, w.x, max(warp - 1, 0)), by = __shfl_sync(0xFFFFFFFFu, w.y, max(warp - 1, 0));
    return {(warp ? bx : 0) + inc.x - v.x, (warp ? by : 0) + inc.y - v.y};
}

// One cluster of `size` CTAs per (sequence, KV head), each with a run of its slots: the newest position,
// then the threshold weight by three passes of a radix select (histograms in shared memory, summed over the
// cluster by every CTA for itself), then the lists. A slot's order and position are read from memory once
// and stay in shared memory (CACHED). Ties at the threshold go to the lowest slots: the last histogram says
// how many of them each CTA holds. holes: [B * Hkv][budget] scratch, the freed slots in order. Bound by
// latency: seven cluster barriers and about as many block scans, 31 us for 16 x 2 lists of 20,000 to 32,768
// slots (7 MB). One CTA to a list took 58 us (the atomics on one SM's shared memory).
template <bool CACHED>
__global__ void __launch_bounds__(kThreads) k_evict_select(const Cache4EvictArgs a, int32_t *holes, int size)
{
    extern __shared__ uint2 slots[];  // CACHED: (order, position)
    __shared__ Exchange ex;
    __shared__ Pair part[kWarps];
    __shared__ int sh_digit, sh_need;
    after_last();
    const int bh = blockIdx.x / size, rank = blockIdx.x % size, b = bh / a.src.Hkv, tid = threadIdx.x;
    const int len = max(0, (int)min((int64_t)a.src.length[b], a.src.cap));
    const int left = min(len, a.budget);
    const float *weight = a.src.weight + bh * a.src.cap;
    const int32_t *pos = a.src.pos + bh * a.src.cap;
    int32_t *kept = a.kept + (int64_t)bh * a.budget;
    holes += (int64_t)bh * a.budget;
    if (len <= a.budget) {
        for (int j = rank * kThreads + tid; j < a.budget; j += size * kThreads) kept[j] = j < len ? j : -1;
        return;
    }
    // this CTA's slots: c0 .. c0 + n - 1
    const int per = (len + size - 1) / size, c0 = min(len, rank * per), n = min(len, c0 + per) - c0;
    for (int i = tid; i < kPasses * kBins; i += kThreads) (&ex.hist[0][0])[i] = 0u;
    if (tid == 0) {
        ex.newest = INT32_MIN;
        ex.recent = 0;
    }
    __syncthreads();
    int newest = INT32_MIN;
#pragma unroll 4
    for (int i = tid; i < n; i += kThreads) {
        const int p = pos[c0 + i];
        if (CACHED) slots[i] = make_uint2(order_of(weight[c0 + i]), (uint32_t)p);
        newest = max(newest, p);
    }
    newest = __reduce_max_sync(0xFFFFFFFFu, newest);
    if ((tid & 31) == 0) atomicMax(&ex.newest, newest);
    auto slot_at = [&](int i) -> uint2 { return CACHED ? slots[i] : make_uint2(order_of(weight[c0 + i]), (uint32_t)pos[c0 + i]); };
    cluster_sync();
    newest = INT32_MIN;
    for (int r = 0; r < size; ++r) newest = max(newest, (int)ld_cluster(&ex.newest, r));
    const int64_t line = (int64_t)newest - a.recent;  // newer than this: recent
    auto is_recent = [&](uint2 s) { return (int64_t)(int32_t)s.y > line; };

    // the first histogram, of the slots that are not recent, and how many are
    int mine = 0;
    for (int i = tid; i < n; i += kThreads) {
        const uint2 s = slot_at(i);
        if (is_recent(s))
            ++mine;
        else
            atomicAdd(&ex.hist[0][s.x >> 21], 1u);
    }
    mine = __reduce_add_sync(0xFFFFFFFFu, mine);
    if ((tid & 31) == 0 && mine > 0) atomicAdd(&ex.recent, mine);
    cluster_sync();
    int n_recent = 0;
    for (int r = 0; r < size; ++r) n_recent += (int)ld_cluster(&ex.recent, r);
    // the threshold lies among the others (recent slots all stay), or where those are too many among the recent
    const bool among_recent = n_recent >= a.budget;
    int need = among_recent ? a.budget : a.budget - n_recent;  // slots to take of that class
    if (among_recent) {
        cluster_sync();  // (the histogram is built again: nobody reads the first one any more)
        for (int i = tid; i < kBins; i += kThreads) ex.hist[0][i] = 0u;
        __syncthreads();
        for (int i = tid; i < n; i += kThreads) {
            const uint2 s = slot_at(i);
            if (is_recent(s)) atomicAdd(&ex.hist[0][s.x >> 21], 1u);
        }
        cluster_sync();
    }
    uint32_t prefix = 0;
    int ties_before = 0;  // ties in the CTAs before this one
#pragma unroll 1
    for (int pass = 0; pass < kPasses; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
        if (pass > 0) {
            const int above = pass == 1 ? 21 : 10, bits = pass == 1 ? 0x7FF : 0x3FF;
            for (int i = tid; i < n; i += kThreads) {
                const uint2 s = slot_at(i);
                if (is_recent(s) == among_recent && s.x >> above == prefix >> above) atomicAdd(&ex.hist[pass][(s.x >> shift) & bits], 1u);
            }
            cluster_sync();
        }
        // The cluster's histogram: each CTA adds up its share of the bins over the CTAs, then takes all
        // shares. (All of every CTA's bins by every CTA is size times the traffic: 8 CTAs of 4,096 slots 97
        // us instead of 31.)
        const int share = kBins / size;
        if (size > 1) {
            for (int i = tid; i < share; i += kThreads) {
                uint32_t x[kMaxCluster];
#pragma unroll
                for (int r = 0; r < kMaxCluster; ++r) x[r] = r < size ? ld_cluster(&ex.hist[pass][rank * share + i], r) : 0u;
#pragma unroll
                for (int r = 1; r < kMaxCluster; ++r) x[0] += x[r];
                ex.sums[rank * share + i] = x[0];
            }
            cluster_sync();
        }
        // bins from the top: thread t takes PB of them
        constexpr int PB = kBins / kThreads;
        int cnt[PB], sum = 0;
#pragma unroll
        for (int e = 0; e < PB; ++e) {
            const int bin = kBins - 1 - PB * tid - e;
            cnt[e] = (int)(size > 1 ? ld_cluster(&ex.sums[bin], bin / share) : ex.hist[pass][bin]);
        }
#pragma unroll
        for (int e = 0; e < PB; ++e) sum += cnt[e];
        Pair total;
        int before = block_scan({sum, 0}, total, part).x;
#pragma unroll
        for (int e = 0; e < PB; ++e) {
            if (before < need && need <= before + cnt[e]) {
                sh_digit = kBins - 1 - PB * tid - e;
                sh_need = need - before;
            }
            before += cnt[e];
        }
        __syncthreads();
        prefix |= (uint32_t)sh_digit << shift;
        need = sh_need;
        if (pass == kPasses - 1)
            for (int r = 0; r < rank; ++r) ties_before += (int)ld_cluster(&ex.hist[pass][sh_digit], r);
        __syncthreads();
    }

    // Slots above the threshold stay, and of those at it the first `need`. A thread takes a run of slots.
    const int run = (n + kThreads - 1) / kThreads, i0 = min(n, tid * run), i1 = min(n, i0 + run);
    auto state = [&](uint2 s) { return is_recent(s) != among_recent ? (is_recent(s) ? 2 : 0) : s.x > prefix ? 2 : s.x == prefix ? 1 : 0; };
    Pair total;
    int ties = 0;
    for (int i = i0; i < i1; ++i) ties += state(slot_at(i)) == 1;
    const int ties_at = ties_before + block_scan({ties, 0}, total, part).x;
    Pair own = {0, 0};
    int t = ties_at;
    for (int i = i0; i < i1; ++i) {
        const int st = state(slot_at(i));
        const bool keep = st == 2 || (st == 1 && t++ < need);
        if (c0 + i < left)
            own.x += !keep;
        else
            own.y += keep;
    }
    Pair at = block_scan(own, total, part);
    if (tid == 0) {
        ex.holes = total.x;
        ex.movers = total.y;
    }
    cluster_sync();
    for (int r = 0; r < rank; ++r) {
        at.x += (int)ld_cluster(&ex.holes, r);
        at.y += (int)ld_cluster(&ex.movers, r);
    }
    t = ties_at;
    int hole = at.x;
    for (int i = i0; i < i1 && c0 + i < left; ++i) {
        const int st = state(slot_at(i));
        if (st == 2 || (st == 1 && t++ < need))
            kept[c0 + i] = c0 + i;
        else
            holes[hole++] = c0 + i;
    }
    cluster_sync();  // every freed slot of the list is written
    t = ties_at;
    int mover = at.y;
    for (int i = i0; i < i1; ++i) {
        const int st = state(slot_at(i));
        const bool keep = st == 2 || (st == 1 && t++ < need);
        if (keep && c0 + i >= left) kept[__ldcg(&holes[mover++])] = c0 + i;
    }
}

// Moves the rows: four lanes to a slot of the target. In place only what moves. Bound by HBM: a row's
// codes, scales, position and weight are read once and written once, though the pieces of a row that is not
// next to the last one are parts of 32-byte sectors (256 bytes fetched for 152 at head dim 128). One slot
// to a thread, so that the launch has threads enough to keep the loads in flight: 54 us an eviction of 16 x
// 2 lists of 20,000 to 32,768 slots to 8,192 (on a board where it took 51, two slots took 53, which is
// within what boards differ, and four 60).
constexpr int kMoveThreads = 256, kMoveSlots = kMoveThreads / 4;
template <int D>
__global__ void __launch_bounds__(kMoveThreads) k_evict_move(const Cache4EvictArgs a, int blocks)
{
    constexpr int PIECES = D / 32 / 2;  // 16-byte pieces of a row's codes, two lanes for the keys, two for the values
    const int bh = blockIdx.x / blocks, u = threadIdx.x & 3, j = (blockIdx.x - bh * blocks) * kMoveSlots + threadIdx.x / 4;
    // (nothing that the select kernel reads or writes is touched before it has finished)
    after_last();
    const int from = j < a.budget ? a.kept[(int64_t)bh * a.budget + j] : -1;
    if (from >= 0 && !(a.in_place && from == j)) {
        const int64_t rs = bh * a.src.cap + from, rd = bh * a.dst.cap + j;
        const bool values = u >= 2;
        const uint4 *sc = reinterpret_cast<const uint4 *>(values ? a.src.v : a.src.k) + rs * (2 * PIECES) + (u & 1) * PIECES;
        uint4 *dc = reinterpret_cast<uint4 *>(values ? a.dst.v : a.dst.k) + rd * (2 * PIECES) + (u & 1) * PIECES;
        uint4 x[PIECES];
#pragma unroll
        for (int p = 0; p < PIECES; ++p) x[p] = sc[p];
        // lane 0: key scales; 1: weight; 2: value scales; 3: position
        if (u == 0 || u == 2) {
            const uint32_t *p = reinterpret_cast<const uint32_t *>(values ? a.src.v_scale : a.src.k_scale) + rs * (D / 64);
            uint32_t *q = reinterpret_cast<uint32_t *>(values ? a.dst.v_scale : a.dst.k_scale) + rd * (D / 64);
            uint32_t y[D / 64];
#pragma unroll
            for (int g = 0; g < D / 64; ++g) y[g] = p[g];
#pragma unroll
            for (int g = 0; g < D / 64; ++g) q[g] = y[g];
        } else if (u == 1) {
            a.dst.weight[rd] = a.src.weight[rs];
        } else {
            a.dst.pos[rd] = a.src.pos[rs];
        }
#pragma unroll
        for (int p = 0; p < PIECES; ++p) dc[p] = x[p];
    }
    if (blockIdx.x == 0)  // (nobody reads the lengths any more)
        for (int b = threadIdx.x; b < a.src.B; b += kMoveThreads)
            a.dst.length[b] = max(0, min((int)min((int64_t)a.src.length[b], a.src.cap), a.budget));
}

template <bool CACHED>
cudaError_t launch_select(const Cache4EvictArgs &a, int32_t *holes, int size, size_t bytes, cudaStream_t s)
{
    static Once once;
    const cudaError_t ready = once([] {
        return CACHED ? cudaFuncSetAttribute(k_evict_select<CACHED>, cudaFuncAttributeMaxDynamicSharedMemorySize, kCachedSlots * (int)sizeof(uint2))
                      : cudaSuccess;
    });
    if (ready != cudaSuccess) return ready;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.src.B * a.src.Hkv * size));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = size;
    at[0].val.clusterDim.y = 1;
    at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, k_evict_select<CACHED>, a, holes, size);
    note_launch();
    return e;
}

template <int D>
cudaError_t launch_move(const Cache4EvictArgs &a, cudaStream_t s)
{
    const int blocks = (a.budget + kMoveSlots - 1) / kMoveSlots;
    return launch_chained(k_evict_move<D>, dim3((unsigned)((int64_t)blocks * a.src.B * a.src.Hkv)), dim3(kMoveThreads), 0, s, a, blocks);
}

}  // namespace

cudaError_t launch_cache4_evict(const Cache4EvictArgs &a, int32_t *holes, cudaStream_t s)
{
    // CTAs of a list: so many that a thread has at most eight slots, up to the cluster's limit
    int size = 1;
    while (size < kMaxCluster && (int64_t)size * kThreads * 8 < a.src.cap) size *= 2;
    const int64_t per = (a.src.cap + size - 1) / size;
    cudaError_t e = per <= kCachedSlots ? launch_select<true>(a, holes, size, (size_t)per * sizeof(uint2), s)
                                        : launch_select<false>(a, holes, size, 0, s);
    if (e != cudaSuccess) return e;
    e = a.src.D == 128 ? launch_move<128>(a, s) : launch_move<64>(a, s);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace ris
