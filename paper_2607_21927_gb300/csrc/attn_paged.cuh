// How attention over pages is shared out, for both of its kernels.
//
// A row tile is a sequence's next `tokens` new tokens x a block of the query heads of a KV head (row r is
// token r / block, head r % block), so that a token's heads share every key they read. It sees the keys
// from the first that its first row sees up to its last row's own, and the first `anchors`: a list of granules
// (32 keys; in fp32 a tile), those of the anchors first, cut into n tiles of BN keys, and the row tile costs n and
// as many tiles more as beginning and ending it take: 5 in bf16 at head dim 128 (16,384 rows at 12 / 2 heads: 556 us when it
// was chosen, 542 now; with 4 580, with 3 643, as the CTAs that have the short row tiles come last), 3 at 64 (16,384 rows at 32 / 4
// heads: 1,064 us, now 1,056; with 5 1,074), 1 in fp32 (900 rows: 156 us, with 4 186). The row tiles of all sequences, heads innermost,
// laid one after another make a line of that length, which is cut into as many equal runs as there are
// CTAs: one row against 60,000 keys and 8,000 rows against 30,000 are spread over the SMs alike, whatever
// the lengths, which only the device knows. A row tile that lies in one run is finished there; of the
// others each run leaves a part (its reference, sum and product), and k_paged_join adds these up in the
// order of the runs. Nothing depends on the order in which CTAs run.
#pragma once

#include <cstdint>

#include "serve.h"

namespace ris {
namespace paged {

// 0 <= length <= reach
__device__ __forceinline__ int length_of(const PagedAttendArgs &a, int seq) { return min(max(a.c.length[seq], 0), a.reach); }

// What a row tile sees, in granules: `sinks` from key 0 on, then those from granule `first` up to key `end`; n tiles.
template <int BN>
constexpr int kGranule = BN == kPagedTileKeys ? kPagedGranule : BN;
struct Sight {
    int pos0;   // position of its first row (negative: it is before the sequence's first slot)
    int tokens;
    int low, end;  // keys [low, end) and [0, anchors) are seen by some row
    int sinks, first, n;
    __device__ __forceinline__ int granule(int g) const { return g < sinks ? g : first + g - sinks; }
};
template <int BN>
__device__ __forceinline__ Sight sight_of(const PagedAttendArgs &a, int length, int rows, int tile)
{
    Sight s;
    const int t0 = tile * a.tokens;
    s.tokens = min(a.tokens, rows - t0);
    s.pos0 = length - rows + t0;
    s.end = max(0, s.pos0 + s.tokens);
    s.low = a.window == 0 ? 0 : max(0, max(s.pos0, 0) - (a.window - 1));
    constexpr int GR = kGranule<BN>, OF = BN / GR;  // of a tile
    s.first = s.low / GR;
    s.sinks = s.end > 0 ? min((min(a.anchors, s.end) + GR - 1) / GR, s.first) : 0;
    s.n = s.end > 0 ? (s.sinks + (s.end + GR - 1) / GR - s.first + OF - 1) / OF : 0;
    return s;
}
// whether the row at `pos` sees key j
__device__ __forceinline__ bool sees(const PagedAttendArgs &a, int pos, int j)
{
    return j <= pos && (a.window == 0 || pos - j < a.window || j < a.anchors);
}

// A sequence's cost where it has one row tile (0 without rows).
template <int BN>
__device__ __forceinline__ int seq_cost(const PagedAttendArgs &a, int seq)
{
    const int rows = a.off[seq + 1] - a.off[seq];
    return rows > 0 ? sight_of<BN>(a, length_of(a, seq), rows, 0).n + a.unit_cost : 0;
}

__device__ __forceinline__ int64_t warp_scan(int64_t x)
{
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(0xFFFFFFFFu, x, o);
        if ((threadIdx.x & 31) >= o) x += y;
    }
    return x;
}
// Exclusive sum over the block's threads; all = the whole sum. `mem`: THREADS / 32 words.
template <int THREADS>
__device__ __forceinline__ int64_t block_scan(int64_t x, int64_t *mem, int64_t &all)
{
    const int64_t in = warp_scan(x);
    __syncthreads();
    if ((threadIdx.x & 31) == 31) mem[threadIdx.x >> 5] = in;
    __syncthreads();
    int64_t before = 0;
    all = 0;
#pragma unroll 8
    for (int w = 0; w < THREADS / 32; ++w) {
        const int64_t y = mem[w];
        before += w < (int)(threadIdx.x >> 5) ? y : 0;
        all += y;
    }
    return before + in - x;
}

// The part of the line that a CTA takes.
struct Run {
    int64_t v0, v1;     // its ends
    int64_t total;      // the line's length
    int64_t u0;         // where its first item begins
    int item;           // which that is
    int runs;           // as many as are used
    __device__ __forceinline__ int64_t begin(int c) const { return total / runs * c + total % runs * c / runs; }
};
struct RunMem {
    int64_t sums[32];
    int64_t u0;
    int item;
    Run run;  // (a place for the caller's copy)
};
template <int BN, int THREADS>
__device__ __forceinline__ Run run_of(const PagedAttendArgs &a, int cta, RunMem &mem)
{
    Run r{};
    const int units = a.c.Hkv * a.blocks;  // row tiles of an item
    auto use = [&](int64_t cost) {
        r.total = cost * units;
        r.runs = (int)min((int64_t)a.runs, max((int64_t)1, r.total));
        if (cta < r.runs && r.total > 0) r.v0 = r.begin(cta), r.v1 = r.begin(cta + 1);
    };
    if (a.max_items > 0) {
        const int n = *a.n_items;
        use(a.prefix[n]);
        // the last item that begins at or before v0 (each has a cost)
        int lo = 0, left = n;
        while (left > 1) {
            const int step = (left + THREADS - 1) / THREADS, i = lo + (int)threadIdx.x * step;
            const int k = __syncthreads_count((int)threadIdx.x * step < left && a.prefix[i] * units <= r.v0);
            left = min(step, left - (k - 1) * step);
            lo += (k - 1) * step;
        }
        r.item = lo;
        r.u0 = n > 0 ? a.prefix[lo] * units : 0;
        return r;
    }
    const int B = a.c.B;
    int64_t cost = 0, all, mine = 0;
    for (int s0 = 0; s0 < B; s0 += THREADS) {
        const int s = s0 + threadIdx.x;
        mine = s < B ? seq_cost<BN>(a, s) : 0;
        block_scan<THREADS>(mine, mem.sums, all);
        cost += all;
    }
    use(cost);
    if (r.v0 >= r.v1) return r;
    int64_t before = 0;
    for (int s0 = 0; s0 < B; s0 += THREADS) {
        const int s = s0 + threadIdx.x;
        if (B > THREADS) mine = s < B ? seq_cost<BN>(a, s) : 0;
        const int64_t at = (before + block_scan<THREADS>(mine, mem.sums, all)) * units;
        if (mine > 0 && at <= r.v0 && r.v0 < at + mine * units) mem.u0 = at, mem.item = s;
        before += all;
    }
    __syncthreads();
    r.u0 = mem.u0;
    r.item = mem.item;
    return r;
}

// A run's part of a row tile.
struct Unit {
    Sight sight;
    int j0, j1;      // key tiles of the part
    int seq, head0, heads, kv_head;
    int row0;        // its first row in q / out
    int part;        // where the part goes, -1: it is the whole row tile
    PagedSplit split;  // first = -1: nothing for the join to do on this run's account
};
struct Walk {
    int64_t v, u0;
    int item, unit, cost;  // cost 0: the item has not been looked at
    int seq, row0;
    Sight sight;
    Walk() = default;
    __device__ __forceinline__ explicit Walk(const Run &r) : v(r.v0), u0(r.u0), item(r.item), unit(0), cost(0), seq(0), row0(0) {}
    template <int BN>
    __device__ __forceinline__ bool next(const PagedAttendArgs &a, const Run &r, Unit &x)
    {
        const int units = a.c.Hkv * a.blocks;
        while (v < r.v1) {
            if (cost == 0) {
                PagedItem it{item, 0};
                if (a.max_items > 0) it = a.items[item];
                const int off = a.off[it.seq], rows = a.off[it.seq + 1] - off;
                if (rows == 0) {
                    ++item;
                    continue;
                }
                sight = sight_of<BN>(a, length_of(a, it.seq), rows, it.tile);
                cost = sight.n + a.unit_cost;
                seq = it.seq;
                row0 = off + it.tile * a.tokens;
                unit = 0;
                if (v > u0) {  // a run's first item
                    unit = (int)((v - u0) / cost);
                    u0 += (int64_t)unit * cost;
                }
            }
            const int64_t at = u0;
            const int n = sight.n, j0 = (int)(v - at), j1 = (int)min((int64_t)n, r.v1 - at), u = unit;
            v = u0 = at + cost;
            const bool last_of_item = ++unit == units;
            x.sight = sight;
            x.seq = seq;
            x.row0 = row0;
            if (last_of_item) cost = 0, ++item;
            if (n > 0 ? j0 >= j1 : j0 > 0) continue;
            x.j0 = j0;
            x.j1 = max(j0, j1);
            x.kv_head = u / a.blocks;
            const int b = u % a.blocks;
            x.head0 = x.kv_head * a.G + b * a.block;
            x.heads = min(a.block, a.G - b * a.block);
            const bool begins = at >= r.v0, ends = at + n <= r.v1;
            x.part = n == 0 || (begins && ends) ? -1 : 2 * (int)blockIdx.x + (begins ? 1 : 0);
            x.split.first = -1;
            if (begins && !ends) {
                int c = blockIdx.x;
                while (r.begin(c + 1) < at + n) ++c;
                x.split = PagedSplit{(int)blockIdx.x, c, row0, sight.tokens, x.head0, x.heads, {}};
            }
            return true;
        }
        return false;
    }
};

// Where key j of sequence seq lies, in elements from the pool's start (of its KV head's rows); -1 for an
// entry that is no page.
__device__ __forceinline__ int page_of(const PagedArgs &c, int seq, int j)
{
    const int p = c.table[(int64_t)seq * c.table_len + (j >> c.page_log2)];
    return p >= 0 && p < c.n_pages ? p : -1;
}
__device__ __forceinline__ int64_t slot_at(const PagedArgs &c, int page, int head, int j)
{
    return (int64_t)page * c.page_stride + (int64_t)head * c.head_stride + (int64_t)(j & ((1 << c.page_log2) - 1)) * c.slot_stride;
}

}  // namespace paged
}  // namespace ris
