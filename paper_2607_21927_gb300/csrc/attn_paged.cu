// Attention over pages on the 5th-generation tensor cores, bf16: from one token against a long cache to a
// chunk of a prompt.
//
// S = Q K^T with bf16 operands (exact products, fp32 sums), one online softmax per row, O = P V with P
// rounded to bf16 (2^-8 of a weight at most: as much as the bf16 output's own rounding, averaged over the
// keys; values cannot be converted to fp16 ahead of a call, as that would read the whole cache) and the
// row's sum from the fp32 weights. The heads of a KV head share a row tile (attn_paged.cuh), so few rows
// read a key once for all of them.
//
// Persistent, each CTA on its run of the line, one row tile at a time:
//   head dim 128  one CTA to an SM (TMEM 512 columns), two softmax groups that take the row tile's key tiles in turn and add
//                 their weights up in one O, three buffers of scores. 8,192 rows behind 24,576 keys at 12 / 2 heads take 885 us
//                 (1.6 PFLOP/s; 985 in a long row of calls, at the power limit): a tile takes 1,350 cycles, of which shared
//                 memory is busy for 1,280 (Q and K read for the scores, V for the outputs, 64 KB written by TMA). With one group and two
//                 buffers 1,015, with two CTAs of a group and a buffer each 1,130. 16 single tokens behind 48 to 64 thousand keys: 138 us, 96%
//                 of the copy rate.
//   head dim 64   two CTAs to an SM (TMEM 256 columns) with a group each, weights beside the scores; nothing is full, a softmax warp's
//                 chain of 2,370 cycles a tile sets the time: 16,384 rows at 32 / 4 heads take 1,056 us; one CTA took 1,650.
// The first warps (a group's four) do the softmax, one thread per row; a warp without a row only passes the tiles on. Then
//   kLoadQK   the run's units, query and key tiles, kLoadV value tiles: TMA, a box for each page of a tile, the
//             boxes of a tile issued by as many lanes; a page that no row sees is asked for past the pool's end, which
//             fills its place with zeros;
//   kScores   S = Q K^T as soon as its columns are free, and the last warp O += P V.
//
// A product over a tile multiplies keys that a row does not see by 0, and 0 times an infinity is not 0. The
// slots past the last row's own key, where a page may hold anything, are cleared in the tile by the softmax
// warps. Where a row comes out not finite all the same (it sees a key that holds an infinity or NaN, or only other rows
// of its tile do), or has outgrown its reference, the CTA goes through its run a second time: values that are not finite, of keys that not all
// rows of a unit see, are taken out of the tiles and added to the rows that see them at the end, and a row that outgrew its reference
// begins with its largest score. 2,048 rows behind 6,144 keys at 12 / 2 heads of 128 take 89 us, 160 to 225 with a NaN in a key that all of them
// see, in one in their middle or in 300 of them (90 ms when each row that was not finite was computed again by itself); single tokens beside them whose
// scores grow without bound 135 (11 ms).
//
// Every mbarrier wait is bounded; a wait that gives up sets the device error word, every role falls through
// to the end, TMEM is released and the CTA returns.
#include <cuda.h>
#include <cuda_bf16.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "attn_common.cuh"
#include "attn_paged.cuh"
#include "row_tiles.cuh"

namespace ris {

// Device error words of this file, read by ris_device_status: a bounded wait gave up; a key outside the pages.
__device__ unsigned int g_ris_paged_wait, g_ris_paged_page;

namespace {

using namespace tc;
using namespace paged;

constexpr int BM = kTileRows, BN = kTileKeys, GR = kPagedGranule;
static_assert(kPagedTileRows == BM && kPagedTileKeys == BN, "as the work is shared out");
constexpr int kGroupWarps = 4;  // of the softmax group: one thread per row
// The exponent of a weight is rounded once, the reference behind it was rounded as a product: rows that pass
// this (no model's do) are computed again in fp32, where both are rounded alike.
constexpr float kFarLog2 = 0x1p28f;
// A row's reference is its largest score in the first tile of the part where it sees a key, and stays: O is never rescaled, and two
// groups can add to one. Weights may grow by 2^100 above it, which bf16 and fp32 hold with values up to 2^20; rows that pass this need the
// second pass, in which the reference is their largest score. A reference that followed the largest score (by 2^7 at most behind) took 220 us instead of 211
// for the 16,233 ragged rows at 32 / 4 heads of 64 through a window, although it moved in few tiles.
constexpr float kGrowthLog2 = 100.f;
// A row that is not finite, of weights up to 2^24 only, is so for its values: its sums stay below 2^128 with values up to 2^74 at any length.
constexpr float kSureLog2 = 24.f;

// What two softmax groups tell each other.
struct Share {
    float ref[kTileRows];                          // the rows' references
    int done[2][kGroupWarps];                      // each warp's tiles whose references are settled
    float4 sums[2][2][kTileRows];                  // [unit with keys mod 2][group]: sum, its correction, largest score, reference
};

template <int D>
struct Lay {
    static constexpr int CTAS = paged_tile_ctas(D);        // of an SM
    static constexpr int NB = D / 64;                      // 64-column blocks
    // NG softmax groups, which take the tiles of a part in turn; NS buffers of scores; a tile's weights take the place of its
    // scores, or one place beside them
    static constexpr int NG = D == 64 ? 1 : 2, NS = D == 64 ? 1 : 3;
    static constexpr bool OVER = D == 128;
    static constexpr int NSK = D == 64 ? 4 : 3, NSV = 2, NI = 4;
    static constexpr int BLK = 128 * 128, TILE = NB * BLK;  // 128 rows or keys of D 16-bit values
    static constexpr int OFF_K = 0, OFF_V = OFF_K + NSK * TILE, OFF_Q = OFF_V + NSV * TILE, OFF_BARS = OFF_Q + TILE,
                         OFF_INFO = OFF_BARS + 256, OFF_RUN = OFF_INFO + NI * 64,
                         OFF_TMEM = OFF_RUN + (int)sizeof(RunMem), OFF_SHARE = (OFF_TMEM + 8 + 15) / 16 * 16, BYTES = OFF_SHARE + (NG == 1 ? 0 : (int)sizeof(Share));
    // Barriers, of a ring stage:
    //   K_FULL, V_FULL, Q_FULL  its keys / values / the query tile have landed
    //   K_FREE, V_FREE, Q_FREE  the products that read it are done
    //   I_FULL, I_FREE          a unit's description is there / every role has read it
    // and one phase per key tile, of its buffer (tile mod NS):
    //   S_GO    the last scores have been read out of their buffer (only where P has its own columns:
    //           else the value product before has to be done, which says that too)
    //   S_FULL  the next are there
    //   P_GO    P is written
    //   PV_DONE O has settled, P's buffer is free
    // and, of two groups, one phase per unit with keys:
    //   SUMS    every softmax warp has left its rows' sums for the other group
    //   O_FREE  every softmax warp has read its part of O
    // No phase of a barrier is completed before everyone has seen the one before it: scores into a buffer wait for the value
    // product over its last weights, and these for every softmax warp.
    static constexpr int B_K_FULL = 0, B_V_FULL = B_K_FULL + NSK, B_Q_FULL = B_V_FULL + NSV, B_K_FREE = B_Q_FULL + 1,
                         B_V_FREE = B_K_FREE + NSK, B_Q_FREE = B_V_FREE + NSV, B_I_FULL = B_Q_FREE + 1, B_I_FREE = B_I_FULL + NI,
                         B_S_GO = B_I_FREE + NI, B_S_FULL = B_S_GO + 1, B_P_GO = B_S_FULL + NS, B_PV_DONE = B_P_GO + NS,
                         B_SUMS = B_PV_DONE + NS, B_O_FREE = B_SUMS + 1, NBAR = B_PV_DONE + NS + (NG == 1 ? 0 : 2);
    static_assert(8 * NBAR <= OFF_INFO - OFF_BARS && CTAS * (BYTES + 1024) <= 228 * 1024, "barriers; the CTAs of an SM");
    static constexpr uint32_t COLS = 512 / CTAS, T_P = OVER ? 0 : BN, T_O = NS * BN + (OVER ? 0 : BN / 2);  // TMEM; S at 0
    static_assert(T_O + D <= COLS, "TMEM columns");
    // Registers per thread: at launch, then after setmaxnreg of a softmax and of another thread. Shared memory leaves
    // next to no L1, so what a loader spills comes from L2: with 56 for them, single tokens against long caches ran at 5.3
    // TB/s instead of 6.5.
    static constexpr int THREADS = 32 * kGroupWarps * (NG + 1), REGS = NG == 1 ? 128 : 168, SOFTMAX_REGS = 192, OTHER_REGS = (NG + 1) * REGS - NG * SOFTMAX_REGS;
    static_assert(OTHER_REGS % 8 == 0 && THREADS * REGS * CTAS <= 64 * 1024, "the shares of the warpgroups add up to the launch's, within the SM's");
};

// What the roles need to know of a unit.
struct Info {
    int n;              // key tiles of this part, -1: no more units
    int j0, sinks, first;  // the first of them; which keys the granules hold (Sight)
    int pos0, tokens, low, end;
    int head0, heads, kv_head, seq, row0, part;
    // the key of a column of the part's tile j
    __device__ __forceinline__ int key(int j, int col) const
    {
        const int g = BN / GR * (j0 + j) + col / GR;
        return GR * (g < sinks ? g : first + g - sinks) + col % GR;
    }
};
static_assert(sizeof(Info) <= 64, "the ring's slots");

// P = 2^(s sc - mu) of columns C0 .. C1 - 1 as bf16, two keys to a word, and the sum of the weights before they
// are rounded
template <int C0, int C1>
__device__ __forceinline__ float weights_of(const float (&sv)[BN], float sc, float mu, uint32_t (&hw)[BN / 2])
{
    const uint64_t sc2 = f2_pack(sc, sc), nmu2 = f2_pack(-mu, -mu);
    uint64_t sum[2] = {0, 0};
#pragma unroll
    for (int w = C0 / 2; w < C1 / 2; ++w) {
        float x0, x1;
        f2_unpack(f2_fma(f2_pack(sv[2 * w], sv[2 * w + 1]), sc2, nmu2), x0, x1);
        x0 = ex2(x0);
        x1 = ex2(x1);
        sum[w & 1] = f2_add(sum[w & 1], f2_pack(x0, x1));
        hw[w] = pack_bf16(x0, x1);
    }
    float a, b;
    f2_unpack(f2_add(sum[0], sum[1]), a, b);
    return a + b;
}

// A lane's box of a tile and the table's entry for it.
struct Box {
    int key, entry;
    bool seen;  // by some row
    __device__ __forceinline__ Box(const PagedAttendArgs &a, const Info &x, int j, int col, bool mine) : key(x.key(j, col)), entry(-1)
    {
        seen = mine && key < x.end && (key + a.box_rows > x.low || key < a.anchors);
        if (seen) entry = a.c.table[(int64_t)x.seq * a.c.table_len + (key >> a.c.page_log2)];
    }
    // its page, or n_pages (past the pool's end) for one that no row sees or whose entry is no page
    __device__ __forceinline__ int page(const PagedAttendArgs &a) const
    {
        const bool is = entry >= 0 && entry < a.c.n_pages;
        if (seen && !is) atomicOr(&g_ris_paged_page, 1u);
        return seen && is ? entry : a.c.n_pages;
    }
};

// Keys of a unit, of those before its end: whether all its rows see one, whether any does.
__device__ __forceinline__ bool by_all(const PagedAttendArgs &a, int pos0, int end, int key)
{
    return key <= pos0 && (a.window == 0 || end - 1 - key < a.window || key < a.anchors);
}
__device__ __forceinline__ bool by_any(const PagedAttendArgs &a, int low, int end, int key) { return key < end && (key >= low || key < a.anchors); }

// Bits 15 and 31 where the bf16 halves of a word are not finite.
__device__ __forceinline__ uint32_t not_finite(uint32_t w) { return ((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u; }
// A key's values (row r of a tile) where not all rows of the unit see it, as 0 times an infinity or NaN is not 0: zeros where none does;
// where some do, what is not finite becomes 0 here and is added to their outputs at the end. Whether there was any.
template <int D>
__device__ __noinline__ bool clean_values(const PagedAttendArgs &a, const Info &x, int key, int r, unsigned char *row)
{
    const bool any = by_any(a, x.low, x.end, key);
    bool found = false;
#pragma unroll 2
    for (int e = 0; e < D / 8; ++e) {
        uint4 *const p = reinterpret_cast<uint4 *>(row + (e >> 3) * Lay<D>::BLK + (((e ^ r) & 7) << 4));
        const uint4 y = *p;
        if (any && ((not_finite(y.x) | not_finite(y.y)) | (not_finite(y.z) | not_finite(y.w))) == 0) continue;
        auto kept = [any](uint32_t w) { return any ? w & ~((not_finite(w) >> 15) * 0xFFFFu) : 0u; };
        *p = make_uint4(kept(y.x), kept(y.y), kept(y.z), kept(y.w));
        found = any;
    }
    return found;
}

template <int THREADS>
__device__ __forceinline__ void all_here()  // the softmax warps, after everything else
{
    asm volatile("barrier.cta.sync 1, %0;" ::"n"(THREADS) : "memory");
}

// What is left to do after a second pass, in the place of the tiles.
//  - Values that are not finite, of keys that only some rows of a unit see, went into the products as zeros: they are added to the rows that see
//    them. There are 254 such keys at most, at the edges of a unit.
//  - Rows that are marked even so, of scores that are too large, are computed again in fp32, each key only where the row sees it: a few rows at a time,
//    a granule of 32 keys to a warp. D / 8 lanes share a key, 8 channels to a lane; the scores go by way of shared memory to a lane per key.
constexpr uint32_t kMarked = 0xFFFFFFFFu;  // first word of a half of a marked row (a NaN that no instruction makes); then comes its largest score
template <int D, int WARPS>
struct Rest {
    static constexpr int ROWS = 4, LOADS = 8;  // rows, and loads of a lane, at once
    PagedAttendArgs args;  // (by reference to the kernel's own they would be read from memory at every use)
    Walk walk;
    Unit unit;
    int more, keys;          // whether there is a unit; poisoned keys at its edges
    int key[256];
    uint32_t bits[256][D / 8];  // which of eight channels are NaN (bits 0 to 7), infinity (8 to 15), -infinity (16 to 23)
    uint32_t marked[kTileRows / 32];
    float p[WARPS][ROWS][32];
    float2 ml[WARPS][ROWS];
    float o[WARPS][ROWS][D];
};
static_assert(sizeof(Rest<128, 8>) <= Lay<128>::OFF_BARS && sizeof(Rest<64, 4>) <= Lay<64>::OFF_BARS, "in the place of the tiles");

// where a row of a unit lies in the outputs, or in the unit's part of them
template <int D>
__device__ __forceinline__ int64_t row_at(const PagedAttendArgs &a, const Unit &u, int r)
{
    return u.part < 0 ? ((int64_t)(u.row0 + r / a.block) * a.Hq + u.head0 + r % a.block) * D : ((int64_t)u.part * a.part_rows + r) * D;
}

template <int D, int WARPS>
__device__ __forceinline__ void marked_rows(const PagedAttendArgs &a, Rest<D, WARPS> &sh)
{
    constexpr int C = D / 32, R = Rest<D, WARPS>::ROWS, U = Rest<D, WARPS>::LOADS, T = 32 * WARPS, OF = BN / GR;
    constexpr int KL = D / 8, KP = 32 / KL;  // lanes of a key, keys side by side
    constexpr uint32_t ALL = 0xFFFFFFFFu;
    const Unit &u = sh.unit;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, ch = lane % KL * 8, kg = lane / KL;
    for (int r0 = 0;;) {
        int row[R], n = 0, last = -1;
        for (; r0 < kTileRows && n < R; ++r0) {
            if ((sh.marked[r0 / 32] >> (r0 & 31) & 1) == 0) continue;
#pragma unroll
            for (int k = 0; k < R; ++k) row[k] = k >= n ? r0 : row[k];  // (the rest of the last few: the last one once more)
            ++n;
            last = u.sight.pos0 + r0 / a.block;
        }
        if (n == 0) break;
        uint4 q[R];
        float o[R][8] = {}, m[R], l[R];
#pragma unroll
        for (int k = 0; k < R; ++k) {
            m[k] = -INFINITY, l[k] = 0.f;
            q[k] = *reinterpret_cast<const uint4 *>(reinterpret_cast<const __nv_bfloat16 *>(a.q) + (int64_t)(u.row0 + row[k] / a.block) * a.q_stride +
                                                    (u.head0 + row[k] % a.block) * D + ch);
        }
        auto value = [](const uint4 &x, int e) {
            const uint32_t w = e < 2 ? x.x : e < 4 ? x.y : e < 6 ? x.z : x.w;
            return __uint_as_float(e % 2 ? w & 0xFFFF0000u : w << 16);
        };
        float (&p)[R][32] = sh.p[warp];
#pragma unroll 1
        for (int g = OF * u.j0 + warp; g < OF * u.j1; g += WARPS) {
            const int key0 = GR * u.sight.granule(g);
            if (key0 > last) continue;
            uint32_t seen[R], any = 0;  // keys of the granule, by row
#pragma unroll
            for (int k = 0; k < R; ++k) {
                seen[k] = __ballot_sync(ALL, sees(a, u.sight.pos0 + row[k] / a.block, key0 + lane));
                any |= seen[k];
            }
            if (any == 0) continue;
            const int page = (any >> lane & 1) != 0 ? page_of(a.c, u.seq, key0 + lane) : -1;
            const int64_t at = page >= 0 ? slot_at(a.c, page, u.kv_head, key0 + lane) : -1;
            any = __ballot_sync(ALL, page >= 0);
            // 8 channels of U x KP keys of either pool, zeros for those that no row sees
            auto load = [&](uint4 (&x)[U], const void *pool, int i0) {
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    const int64_t from = __shfl_sync(ALL, at, i0 + i * KP + kg);
                    x[i] = from >= 0 ? *reinterpret_cast<const uint4 *>(reinterpret_cast<const __nv_bfloat16 *>(pool) + from + ch) : make_uint4(0u, 0u, 0u, 0u);
                }
            };
#pragma unroll 1
            for (int i0 = 0; i0 < GR; i0 += U * KP) {
                uint4 x[U];
                load(x, a.c.k, i0);
#pragma unroll
                for (int i = 0; i < U; ++i)
#pragma unroll
                    for (int k = 0; k < R; ++k) {
                        float s = 0.f;
#pragma unroll
                        for (int e = 0; e < 8; ++e) s = fmaf(value(q[k], e), value(x[i], e), s);
#pragma unroll
                        for (int w = KL / 2; w > 0; w >>= 1) s += __shfl_xor_sync(ALL, s, w);
                        if (lane % KL == 0) p[k][i0 + i * KP + kg] = s;
                    }
            }
            __syncwarp();
#pragma unroll
            for (int k = 0; k < R; ++k) {
                seen[k] &= any;
                const bool mine = (seen[k] >> lane & 1) != 0;
                const float s = mine ? __fmul_rn(p[k][lane], a.scale_log2) : -INFINITY;
                const float top = fmaxf(m[k], warp_max(s)), ref = top == -INFINITY ? 0.f : top, al = exp2f(m[k] - ref), w = mine ? exp2f(s - ref) : 0.f;
                m[k] = top;
                l[k] = fmaf(l[k], al, warp_sum(w));
#pragma unroll
                for (int e = 0; e < 8; ++e) o[k][e] *= al;
                p[k][lane] = w;
            }
            __syncwarp();
#pragma unroll 1
            for (int i0 = 0; i0 < GR; i0 += U * KP) {
                uint4 x[U];
                load(x, a.c.v, i0);
#pragma unroll
                for (int i = 0; i < U; ++i)
#pragma unroll
                    for (int k = 0; k < R; ++k) {
                        if ((seen[k] >> (i0 + i * KP + kg) & 1) == 0) continue;
                        const float w = p[k][i0 + i * KP + kg];
#pragma unroll
                        for (int e = 0; e < 8; ++e) o[k][e] = fmaf(w, value(x[i], e), o[k][e]);
                    }
            }
            __syncwarp();
        }
#pragma unroll
        for (int k = 0; k < R; ++k) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float y = o[k][e];
#pragma unroll
                for (int w = KL; w < 32; w <<= 1) y += __shfl_xor_sync(ALL, y, w);
                if (kg == 0) sh.o[warp][k][ch + e] = y;
            }
            if (lane == 0) sh.ml[warp][k] = make_float2(m[k], l[k]);
        }
        all_here<T>();
        if (warp < n) {  // the warps' parts of a row, in order
            int r = 0;
#pragma unroll
            for (int k = 0; k < R; ++k) r = k == warp ? row[k] : r;
            float top = -INFINITY, sum = 0.f, y[C] = {};
            for (int w = 0; w < WARPS; ++w) top = fmaxf(top, sh.ml[w][warp].x);
            const float ref = top == -INFINITY ? 0.f : top;
            for (int w = 0; w < WARPS; ++w) {
                const float f = exp2f(sh.ml[w][warp].x - ref);
                sum = fmaf(sh.ml[w][warp].y, f, sum);
#pragma unroll
                for (int c = 0; c < C; ++c) y[c] = fmaf(sh.o[w][warp][C * lane + c], f, y[c]);
            }
            const int64_t to = row_at<D>(a, u, r) + C * lane;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                if (u.part < 0)
                    reinterpret_cast<__nv_bfloat16 *>(a.out)[to + c] = __float2bfloat16_rn(sum == 0.f ? 0.f : y[c] / sum);
                else
                    a.part_o[to + c] = y[c];
            }
            if (lane == 0) {
                if (u.part >= 0)
                    a.part_ml[(int64_t)u.part * a.part_rows + r] = make_float4(top, sum, sum, 0.f);
                else if (a.lse != nullptr)
                    a.lse[(int64_t)(u.head0 + r % a.block) * a.q_total + u.row0 + r / a.block] = (top + log2f(sum)) * kLn2;
            }
        }
        all_here<T>();
    }
}

template <int D, int WARPS>
__device__ __noinline__ void the_rest(const PagedAttendArgs &args, const Run &run, unsigned char *smem, bool marks)
{
    constexpr int C = D / 32, T = 32 * WARPS, KL = D / 8;  // lanes of a key
    constexpr uint32_t ALL = 0xFFFFFFFFu;
    Rest<D, WARPS> &sh = *reinterpret_cast<Rest<D, WARPS> *>(smem);
    const Unit &u = sh.unit;
    const PagedAttendArgs &a = sh.args;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, ch = lane % KL * 8, kg = lane / KL;
    if (threadIdx.x == 0) sh.args = args, sh.walk = Walk(run);
    all_here<T>();
    while (true) {
        if (threadIdx.x == 0) {
            sh.more = sh.walk.template next<BN>(a, run, sh.unit);
            sh.keys = 0;
        }
        if (threadIdx.x < kTileRows / 32) sh.marked[threadIdx.x] = 0;
        all_here<T>();
        if (!sh.more) break;
        // keys past the first row's own, and those before the last row's window that another row's still holds
        const int pos0 = u.sight.pos0, end = u.sight.end, first[2] = {max(pos0 + 1, 0), max(u.sight.low, a.anchors)};
        const int n0 = max(0, end - first[0]), n1 = a.window == 0 ? 0 : max(0, min(end - 1 - a.window, pos0) - first[1] + 1);
        for (int i0 = 0; i0 < n0 + n1; i0 += T / KL) {
            const int i = i0 + (int)threadIdx.x / KL, key = i < n0 ? first[0] + i : first[1] + i - n0;
            const int page = i < n0 + n1 ? page_of(a.c, u.seq, key) : -1;
            uint4 x = make_uint4(0u, 0u, 0u, 0u);
            if (page >= 0) x = *reinterpret_cast<const uint4 *>(reinterpret_cast<const __nv_bfloat16 *>(a.c.v) + slot_at(a.c, page, u.kv_head, key) + ch);
            const uint32_t v[4] = {x.x, x.y, x.z, x.w};
            const bool found = (not_finite(v[0]) | not_finite(v[1]) | not_finite(v[2]) | not_finite(v[3])) != 0;
            const uint32_t mine = __ballot_sync(ALL, found) >> (KL * kg) & ((1u << KL) - 1u);  // of this key's lanes
            int to = 0;
            if (mine != 0 && lane % KL == 0) to = atomicAdd(&sh.keys, 1);
            to = __shfl_sync(ALL, to, KL * kg);
            if (mine != 0) {
                uint32_t b = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t h = v[e / 2] >> 16 * (e % 2) & 0xFFFFu;
                    b |= ((uint32_t)((h & 0x7FFFu) > 0x7F80u) | (uint32_t)(h == 0x7F80u) << 8 | (uint32_t)(h == 0xFF80u) << 16) << e;
                }
                if (lane % KL == 0) sh.key[to] = key;
                sh.bits[to][lane % KL] = b;
            }
            __syncwarp();
        }
        all_here<T>();
        for (int r = warp; r < kTileRows && marks; r += WARPS) {
            if (r / a.block >= u.sight.tokens || r % a.block >= u.heads) continue;
            const int64_t at = row_at<D>(a, u, r) + C * lane;
            const uint32_t first = u.part < 0 ? *reinterpret_cast<const uint32_t *>(reinterpret_cast<const __nv_bfloat16 *>(a.out) + at) : __float_as_uint(a.part_o[at]);
            if (__any_sync(ALL, lane % 16 == 0 && first == kMarked) && lane == 0) atomicOr(&sh.marked[r / 32], 1u << (r & 31));
        }
        if (marks) all_here<T>();
        const int keys = sh.keys;
        for (int tok = warp; tok < u.sight.tokens && keys > 0; tok += WARPS) {
            uint32_t b = 0;  // of this lane's channels, as above
#pragma unroll 8
            for (int i = 0; i < keys; ++i) b |= sees(a, pos0 + tok, sh.key[i]) ? sh.bits[i][C * lane / 8] : 0u;
            b >>= C * lane % 8;
            if (!__any_sync(ALL, (b & 0x10101u * ((1u << C) - 1u)) != 0)) continue;
#pragma unroll 4
            for (int h = 0; h < u.heads; ++h) {
                const int r = tok * a.block + h;
                if ((sh.marked[r / 32] >> (r & 31) & 1) != 0) continue;  // (to be computed again anyway)
                const int64_t at = row_at<D>(a, u, r) + C * lane;
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    if ((b >> c & 0x10101u) == 0) continue;
                    const float add = (b >> c & 1) != 0 || (b >> c & 0x10100u) == 0x10100u ? NAN : (b >> c & 0x100u) != 0 ? INFINITY : -INFINITY;
                    if (u.part < 0) {
                        __nv_bfloat16 *const y = reinterpret_cast<__nv_bfloat16 *>(a.out) + at + c;
                        *y = __float2bfloat16_rn(add != add ? add : __bfloat162float(*y) + add);
                    } else {
                        a.part_o[at + c] = add != add ? add : a.part_o[at + c] + add;
                    }
                }
            }
        }
        all_here<T>();
        if (marks) marked_rows<D, WARPS>(a, sh);
        all_here<T>();
    }
}

struct Maps {
    CUtensorMap q, k, v;
};

template <int D>
__global__ void __launch_bounds__(Lay<D>::THREADS, Lay<D>::CTAS) k_paged_tiles(const __grid_constant__ PagedAttendArgs a, const __grid_constant__ Maps maps)
{
    using L = Lay<D>;
    constexpr int NG = L::NG, NS = L::NS, NSK = L::NSK, NSV = L::NSV, NI = L::NI, NB = L::NB, TILE = L::TILE;
    constexpr int kSoftmaxWarps = NG * kGroupWarps, kLoadQK = kSoftmaxWarps, kLoadV = kLoadQK + 1, kScores = kLoadV + 1;
    extern __shared__ __align__(1024) unsigned char smem[];
    uint32_t &tmem_base_sh = *reinterpret_cast<uint32_t *>(smem + L::OFF_TMEM);
    const uint32_t sbase = smem_u32(smem);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const unsigned int *const gave_up = &g_ris_paged_wait;
    const long long limit = a.wait_limit;
    auto bar = [&](int i) { return sbase + (uint32_t)(L::OFF_BARS + 8 * i); };

    // 1: a second pass is needed, 2: something is left to do after it, 4: a wait gave up, 8: it is the second pass, 16: rows
    // are marked after that
    volatile uint32_t &wrong = *reinterpret_cast<volatile uint32_t *>(smem + L::OFF_TMEM + 4);
    auto say = [&](uint32_t what) { atomicOr(const_cast<uint32_t *>(&wrong), what); };
    auto set_up = [&] {  // for a pass, by one warp
        for (int i = lane; i < L::NBAR; i += 32) {
            const bool by_group = i == L::B_S_GO || (i >= L::B_P_GO && i < L::B_P_GO + NS), free = i >= L::B_I_FREE && i < L::B_I_FREE + NI;
            mbar_init(bar(i), by_group ? kGroupWarps : free ? kSoftmaxWarps + 3 : NG > 1 && i >= L::B_SUMS ? kSoftmaxWarps : 1);
        }
        if (NG > 1 && lane < 2 * kGroupWarps) (&reinterpret_cast<Share *>(smem + L::OFF_SHARE)->done[0][0])[lane] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    };

    if (warp == kLoadQK) {
        if (lane == 0) wrong = 0;
        set_up();
    } else if (warp == kScores) {
        tmem_alloc<1, L::COLS>(smem_u32(&tmem_base_sh));
    }
    after_last();
    {
        RunMem &mem = *reinterpret_cast<RunMem *>(smem + L::OFF_RUN);
        const Run r = run_of<BN, L::THREADS>(a, blockIdx.x, mem);
        if (threadIdx.x == 0) mem.run = r;
    }
    const Run &run = reinterpret_cast<const RunMem *>(smem + L::OFF_RUN)->run;
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_base_sh;
    bool ok = (sbase & 1023u) == 0u;
    auto wait_all = [&](int i, int parity) -> bool {
        const bool got = __all_sync(0xFFFFFFFFu, mbar_wait<1>(bar(i), parity, gave_up, limit));
        tc_fence_after();
        return got;
    };
    // The same by looking at the barrier where a test asks for short waits: of one role, as every wait would cost short row tiles 8%.
    auto look_all = [&](int i, int parity) -> bool {
        const bool got = __all_sync(0xFFFFFFFFu, mbar_wait<1, false, true>(bar(i), parity, gave_up, limit));
        tc_fence_after();
        return got;
    };
    // a count in shared memory, and a bounded wait until it is `least` (what was written before it was stored is there)
    auto store_count = [&](int *word, int x) { asm volatile("st.release.cta.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(word)), "r"(x) : "memory"); };
    auto wait_count = [&](const int *word, int least) -> bool {
        const uint32_t at = smem_u32(word);
        const long long since = clock64();
        while (true) {
            int x;
            asm volatile("ld.acquire.cta.shared::cta.b32 %0, [%1];" : "=r"(x) : "r"(at) : "memory");
            if (__all_sync(0xFFFFFFFFu, x >= least)) return true;
            const long long waited = clock64() - since;
            const bool over = waited > limit || (waited > (1LL << 20) && *reinterpret_cast<const volatile unsigned int *>(gave_up) != 0u);
            if (__any_sync(0xFFFFFFFFu, over)) return false;
        }
    };
    // description of unit u (a whole warp); its place is given back once every lane has it
    auto unit = [&](int u, Info &x) -> bool {
        if (!__all_sync(0xFFFFFFFFu, mbar_wait<1>(bar(L::B_I_FULL + u % NI), (u / NI) & 1, gave_up, limit))) return false;
        x = *reinterpret_cast<const Info *>(smem + L::OFF_INFO + u % NI * 64);
        __syncwarp();
        mbar_arrive_if(lane == 0, bar(L::B_I_FREE + u % NI));
        return true;
    };

    // Everyone at the end of a pass; whether there is another one.
    // (the roles' code serves both, but the softmax is there twice: as one, with a variable that says which pass it is, 16,233
    // ragged rows at 32 / 4 heads of 64 through a window took 237 us instead of 217, and with it and the handing over of units going on, 228)
    auto another_pass = [&]() -> bool {
        if (!ok) {
            atomicOr(&g_ris_paged_wait, 2u);
            say(4u);
        }
        __syncwarp();
        tc_fence_before();
        asm volatile("barrier.cta.sync 0;" ::: "memory");
        tc_fence_after();
        if (wrong != 1u) return false;
        if (warp == kLoadQK) {  // (all copies, products and waits of the first one are over)
            for (int i = lane; i < L::NBAR; i += 32) asm volatile("mbarrier.inval.shared::cta.b64 [%0];" ::"r"(bar(i)) : "memory");
            __syncwarp();
            set_up();
        }
        __syncwarp();
        asm volatile("barrier.cta.sync 0;" ::: "memory");
        if (warp == kLoadQK && lane == 0) say(8u);
        return true;
    };

    if (warp >= kSoftmaxWarps) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(L::OTHER_REGS));
        // table entries are asked for a tile ahead where there are registers for it (pages of 16 slots at 12 / 2 heads of 128:
        // 16,384 rows in 725 us instead of 772 when it was built, 699 now; at head dim 64 spilled registers cost 2%)
        constexpr bool AHEAD = D == 128;
        const int boxes = BN / a.box_rows;  // of a tile and 64-column block
        const int col = lane % boxes * a.box_rows, blk = lane / boxes, in_page = (1 << a.c.page_log2) - 1;
        do {  // (a pass)
            if (warp == kLoadQK) {
                const uint32_t q_bytes = (uint32_t)(a.block * a.tokens * 128 * NB);
                int nq = 0, nk = 0;  // query and key tiles asked for
                if (lane == 0) a.split[blockIdx.x].first = -1;
                Walk walk(run);
                Unit y;
                bool more = walk.next<BN>(a, run, y);
                for (int u = 0; ok; ++u) {
                    if (u >= NI) ok = __all_sync(0xFFFFFFFFu, mbar_wait<1>(bar(L::B_I_FREE + u % NI), (u / NI - 1) & 1, gave_up, limit));
                    if (!ok) break;
                    const Info z{more ? y.j1 - y.j0 : -1, y.j0, y.sight.sinks, y.sight.first, y.sight.pos0, y.sight.tokens, y.sight.low, y.sight.end,
                                 y.head0, y.heads, y.kv_head, y.seq, y.row0, y.part};
                    if (lane == 0) {
                        *reinterpret_cast<Info *>(smem + L::OFF_INFO + u % NI * 64) = z;
                        if (more && y.split.first >= 0) a.split[blockIdx.x] = y.split;
                        mbar_arrive(bar(L::B_I_FULL + u % NI));
                    }
                    __syncwarp();
                    if (!more) break;
                    // (read from there, to need fewer registers)
                    const Info &x = *reinterpret_cast<const Info *>(smem + L::OFF_INFO + u % NI * 64);
                    const int n = x.n;
                    Box next(a, x, 0, col, AHEAD && blk < NB && n > 0);
                    for (int j = 0; j < n; ++j, ++nk) {
                        const int st = nk % NSK;
                        const Box at = AHEAD ? next : Box(a, x, j, col, blk < NB);
                        if (AHEAD && j + 1 < n) next = Box(a, x, j + 1, col, blk < NB);
                        if (nk >= NSK) ok = __all_sync(0xFFFFFFFFu, mbar_wait<1>(bar(L::B_K_FREE + st), (nk / NSK - 1) & 1, gave_up, limit));
                        if (!ok) break;
                        if (lane == 0) mbar_arrive_expect_tx<1>(bar(L::B_K_FULL + st), TILE);
                        __syncwarp();
                        if (blk < NB && a.debug_no_loads == 0)
                            tma_load_4d(sbase + L::OFF_K + st * TILE + blk * L::BLK + col * 128, &maps.k, 64 * blk, at.key & in_page, x.kv_head, at.page(a),
                                        bar(L::B_K_FULL + st));
                        if (j > 0) continue;
                        if (nq > 0) ok = __all_sync(0xFFFFFFFFu, mbar_wait<1>(bar(L::B_Q_FREE), (nq - 1) & 1, gave_up, limit));
                        if (!ok) {
                            ++nk;
                            break;
                        }
                        if (lane == 0) {
                            mbar_arrive_expect_tx<1>(bar(L::B_Q_FULL), q_bytes);
                            for (int b = 0; b < NB && a.debug_no_loads == 0; ++b) tma_load_3d<1>(sbase + L::OFF_Q + b * L::BLK, &maps.q, 64 * b, x.head0, x.row0, bar(L::B_Q_FULL));
                        }
                        ++nq;
                        more = walk.next<BN>(a, run, y);  // (while these are on their way)
                    }
                    if (n == 0) more = walk.next<BN>(a, run, y);
                }
                if (lane == 0 && a.debug_no_loads == 0) {
                    // nothing of this warp's may still be on its way to shared memory when the CTA ends
                    if (nq > 0) mbar_wait_own<1>(bar(L::B_Q_FULL), (nq - 1) & 1);
                    for (int i = max(0, nk - NSK); i < nk; ++i) mbar_wait_own<1>(bar(L::B_K_FULL + i % NSK), (i / NSK) & 1);
                }
            } else if (warp == kLoadV) {
                int nv = 0;
                for (int u = 0; ok; ++u) {
                    Info x;
                    ok = unit(u, x);
                    if (!ok || x.n < 0) break;
                    Box next(a, x, 0, col, AHEAD && blk < NB && x.n > 0);
                    for (int j = 0; j < x.n; ++j, ++nv) {
                        const int st = nv % NSV;
                        const Box at = AHEAD ? next : Box(a, x, j, col, blk < NB);
                        if (AHEAD && j + 1 < x.n) next = Box(a, x, j + 1, col, blk < NB);
                        if (nv >= NSV) ok = __all_sync(0xFFFFFFFFu, mbar_wait<1>(bar(L::B_V_FREE + st), (nv / NSV - 1) & 1, gave_up, limit));
                        if (!ok) break;
                        if (lane == 0) mbar_arrive_expect_tx<1>(bar(L::B_V_FULL + st), TILE);
                        __syncwarp();
                        if (blk < NB && a.debug_no_loads == 0)
                            tma_load_4d(sbase + L::OFF_V + st * TILE + blk * L::BLK + col * 128, &maps.v, 64 * blk, at.key & in_page, x.kv_head, at.page(a),
                                        bar(L::B_V_FULL + st));
                    }
                }
                if (lane == 0 && a.debug_no_loads == 0)
                    for (int i = max(0, nv - NSV); i < nv; ++i) mbar_wait_own<1>(bar(L::B_V_FULL + i % NSV), (i / NSV) & 1);
            } else if (ok) {
                // The issuing warps, all lanes: trip counts and addresses come out of warp-wide reductions,
                // which leave them in uniform registers; a product whose operands are in the lanes' registers
                // costs more time to issue than to run.
                const uint32_t tb = __reduce_max_sync(0xFFFFFFFFu, tmem);
                int t = 0, nq = 0;  // tiles; units with keys
                for (int u = 0;; ++u) {
                    Info x;
                    ok = unit(u, x);
                    if (!ok) break;
                    const int n = __reduce_max_sync(0xFFFFFFFFu, x.n);
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
                            else if (t >= NS)
                                ok = ok && wait_all(L::B_PV_DONE + t % NS, (t / NS - 1) & 1);
                            if (!ok) break;
                            const uint32_t kd = desc_lo(sbase + L::OFF_K + st * TILE, 16);
                            if (elect_one()) {
#pragma unroll
                                for (int ks = 0; ks < D / 16; ++ks)
                                    tc_mma_ss<1>(tb + t % NS * BN, qd + dstep((ks >> 2) * L::BLK + (ks & 3) * 32), kd + dstep((ks >> 2) * L::BLK + (ks & 3) * 32), ID_S, ks > 0);
                                tc_commit<1>(bar(L::B_S_FULL + t % NS));
                                tc_commit<1>(bar(L::B_K_FREE + st));
                                if (j == n - 1) tc_commit<1>(bar(L::B_Q_FREE));
                            }
                            __syncwarp();
                        }
                    } else {
                        constexpr uint32_t ID_O = idesc_bf16(BM, D, true);
                        if (NG > 1 && nq > 0) ok = look_all(L::B_O_FREE, (nq - 1) & 1);
                        for (int j = 0; j < n && ok; ++j, ++t) {
                            const int st = t % NSV;
                            ok = look_all(L::B_V_FULL + st, (t / NSV) & 1) && look_all(L::B_P_GO + t % NS, (t / NS) & 1);
                            if (!ok) break;
                            const uint32_t vd = desc_lo(sbase + L::OFF_V + st * TILE, L::BLK);
                            if (elect_one()) {
#pragma unroll
                                for (int ks = 0; ks < BN / 16; ++ks)
                                    tc_mma_ts<1>(tb + L::T_O, tb + L::T_P + t % NS * BN + 8 * ks, vd + dstep(ks * 2048), ID_O, ks > 0 || j > 0);
                                tc_commit<1>(bar(L::B_PV_DONE + t % NS));
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
                    for (int i = max(0, t - NS); i < t; ++i) mbar_wait_own<1>(bar(done + i % NS), (i / NS) & 1);
                    for (int i = max(0, t - ring); i < t; ++i) mbar_wait_own<1>(bar(free + i % ring), (i / ring) & 1);
                    if (warp == kScores && nq > 0) mbar_wait_own<1>(bar(L::B_Q_FREE), (nq - 1) & 1);
                }
            }
        } while (another_pass());
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(L::SOFTMAX_REGS));
        const int group = warp / kGroupWarps, quarter = warp % kGroupWarps;
        const int r = threadIdx.x % BM;  // TMEM lane, row of the tile, key of a tile at the edges
        const int tok = r / a.block, head = r - tok * a.block;
        const int tok_first = quarter * 32 / a.block, tok_last = (quarter * 32 + 31) / a.block;  // of the warp
        const uint32_t lane_off = (uint32_t)(quarter * 32) << 16;
        const uint32_t t_o = tmem + L::T_O + lane_off;
        Share &share = *reinterpret_cast<Share *>(smem + L::OFF_SHARE);
        auto softmax = [&](auto second) __attribute__((always_inline)) {
            constexpr bool careful = decltype(second)::value;
            int t0 = 0;          // tiles of the units before
            [[maybe_unused]] int keyed = 0;  // units with keys
            bool there = false;  // the next scores, seen under the last exponentials: a poll takes 200 cycles and more even if they are
            if (!L::OVER && lane == 0) mbar_arrive(bar(L::B_S_GO));
            for (int u = 0; ok; ++u) {
                // (its description stays in its place until the unit is done)
                ok = __all_sync(0xFFFFFFFFu, mbar_wait<1>(bar(L::B_I_FULL + u % NI), (u / NI) & 1, gave_up, limit));
                const Info &x = *reinterpret_cast<const Info *>(smem + L::OFF_INFO + u % NI * 64);
                const int n = x.n;
                if (!ok || n < 0) break;
                const bool valid = tok < x.tokens && head < x.heads;
                const bool idle = !__any_sync(0xFFFFFFFFu, valid);
                const int pos0 = x.pos0, pos = pos0 + tok, end = x.end;
                // A tile's keys follow one another from k0 on, but for granules of the anchors, which the first `mixed` have.
                int k0 = GR * (x.first - x.sinks) + BN * (x.j0 + group);
                const int mixed = (x.sinks + BN / GR - 1) / (BN / GR) - x.j0;
                // row sum, reference, largest score; by how much the largest score's weight is rounded up: the outputs
                // are divided by the sum with that weight as rounded, so that a row whose weight goes to one key is that key's values
                float l = 0.f, m = -INFINITY, top = -INFINITY, up = 0.f;
                if (careful && valid) {  // a marked row's reference: its largest score
                    const int64_t at = x.part < 0 ? ((int64_t)(x.row0 + tok) * a.Hq + x.head0 + head) * D : ((int64_t)x.part * a.part_rows + r) * D;
#pragma unroll
                    for (int h = 0; h < NG; ++h) {
                        const uint2 y = x.part < 0 ? *reinterpret_cast<const uint2 *>(reinterpret_cast<const __nv_bfloat16 *>(a.out) + at + D / NG * h)
                                                   : *reinterpret_cast<const uint2 *>(a.part_o + at + D / NG * h);
                        if (y.x == kMarked) m = __uint_as_float(y.y);
                    }
                }
                for (int j = group; j < n; j += NG, k0 += NG * BN) {
                    const int t = t0 + j, buf = (unsigned)t % NS;
                    // (after a wait that gave up the loop runs on without waiting: fewer branches in it)
                    if (!__all_sync(0xFFFFFFFFu, there) && ok) ok = wait_all(L::B_S_FULL + buf, (unsigned)t / NS & 1);
                    tc_fence_after();
                    const uint32_t t_s = tmem + lane_off + buf * BN, t_p = t_s + L::T_P;
                    if (idle) {
                        there = false;
                        if (!L::OVER) mbar_arrive_if(lane == 0, bar(L::B_S_GO));
                        // (in step with the others: a wait for a phase tells nothing while the one before it is open, and
                        // an arrival ahead of the others' would count for the last tile's P)
                        if (!L::OVER && j > 0 && ok) ok = wait_all(L::B_PV_DONE, (t - 1) & 1);
                    } else {
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
                        if (j < mixed || k0 + BN - 1 > pos0 + tok_first || (a.window != 0 && pos0 + tok_last - k0 >= a.window)) {
                            uint32_t cw[BN / 32];
#pragma unroll
                            for (int e = 0; e < BN / 32; ++e) {
                                const int k = j < mixed ? x.key(j, 32 * e) : k0 + 32 * e;
                                cw[e] = causal_word(pos - k, 0) &
                                        (a.window == 0 ? 0xFFFFFFFFu : ~causal_word(pos - a.window - k, 0) | causal_word(a.anchors - 1 - k, 0));
                            }
#pragma unroll
                            for (int w = 0; w < BN / 32; ++w) {
                                // (an end of what the rows see lies in one or two of a warp's words)
                                if (__all_sync(0xFFFFFFFFu, cw[w] == 0xFFFFFFFFu)) continue;
#pragma unroll
                                for (int e = 0; e < 32; ++e) drop_unless(sv[32 * w + e], cw[w], 1u << e);
                            }
                        }
                        const float raw = valid ? row_max(sv) : -INFINITY, mx = __fmul_rn(raw, a.scale_log2);
                        if constexpr (NG == 1) {
                            m = m == -INFINITY ? mx : m;
                        } else {
                            // (the groups' weights add up in one O: a row without a reference waits for the other group's last tile)
                            if (__any_sync(0xFFFFFFFFu, valid && m == -INFINITY)) {
                                if (j > 0) {
                                    if (ok) ok = wait_count(&share.done[1 - group][quarter], t);
                                    m = share.ref[r];
                                }
                                if (m == -INFINITY) m = mx;
                                share.ref[r] = m;
                            }
                            __syncwarp();
                            if (lane == 0) store_count(&share.done[group][quarter], t + 1);
                        }
                        const float mu = m == -INFINITY ? 0.f : m;
                        uint32_t hw[BN / 2];
                        float sum = weights_of<0, 96>(sv, a.scale_log2, mu, hw);
                        // polled here, the answers are there when the weights are
                        bool settled = true;
                        if (!L::OVER) settled = j == 0 || mbar_test<1>(bar(L::B_PV_DONE), (t - 1) & 1);
                        there = (NG == 1 || j + NG < n) && mbar_test<1>(bar(L::B_S_FULL + (unsigned)(t + NG) % NS), (unsigned)(t + NG) / NS & 1);
                        sum += weights_of<96, BN>(sv, a.scale_log2, mu, hw);
                        l += sum;
                        const float w = ex2(fmaf(raw, a.scale_log2, -mu));
                        up = mx > top ? __bfloat162float(__float2bfloat16_rn(w)) - w : up;
                        top = fmaxf(top, mx);
                        // P's buffer is free once the last value product is done (a unit's first tile: waited for at the end of the
                        // last unit)
                        if (!L::OVER && !__all_sync(0xFFFFFFFFu, settled) && ok) ok = wait_all(L::B_PV_DONE, (t - 1) & 1);
                        tc_fence_after();
                        tmem_st32(t_p, hw);
                        tmem_st32(t_p + 32, hw + 32);
                        tmem_wait_st();
                    }
                    if (j < mixed || k0 + BN > end || careful) {  // (a thread takes a key)
                        // (the values before in this place have been used: the scores came without waiting for that, and the wait for
                        // the values' phase tells nothing while the one before it is open)
                        static_assert(NG == 1 || NSV == 2, "which ones those are");
                        if (NG > 1 && t >= 2 && ok) ok = wait_all(L::B_PV_DONE + (unsigned)(t - 2) % NS, (unsigned)(t - 2) / NS & 1);
                        if (ok) ok = wait_all(L::B_V_FULL + t % NSV, (t / NSV) & 1);
                        const int key = j < mixed ? x.key(j, r) : k0 + r;
                        unsigned char *const row = smem + L::OFF_V + t % NSV * TILE + r * 128;
                        if (ok && key >= end) {
#pragma unroll
                            for (int e = 0; e < 8 * NB; ++e)
                                *reinterpret_cast<uint4 *>(row + (e >> 3) * L::BLK + (((e ^ r) & 7) << 4)) = make_uint4(0u, 0u, 0u, 0u);
                        } else if (ok && careful && !by_all(a, pos0, end, key)) {
                            if (clean_values<D>(a, x, key, r, row)) say(2u);
                        }
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    }
                    tc_fence_before();
                    __syncwarp();
                    mbar_arrive_if(lane == 0, bar(L::B_P_GO + buf));
                }
                if (ok && n > 0) ok = wait_all(L::B_PV_DONE + (unsigned)(t0 + n - 1) % NS, (unsigned)(t0 + n - 1) / NS & 1);
                if constexpr (NG > 1) {
                    there = false;
                    if (n > 0) {
                        float4 *const sums = share.sums[keyed & 1][0];
                        sums[BM * group + r] = make_float4(l, up, top, m);
                        __syncwarp();
                        mbar_arrive_if(lane == 0, bar(L::B_SUMS));
                        if (ok) ok = wait_all(L::B_SUMS, keyed & 1);
                        const float4 y = sums[r], z = sums[BM + r];  // of either group, in this order in both
                        l = y.x + z.x;
                        up = y.z >= z.z ? y.y : z.y;
                        top = fmaxf(y.z, z.z);
                        m = fmaxf(y.w, z.w);  // (the same, or one of them saw no key)
                        ++keyed;
                    }
                }
                t0 += max(n, 0);
                if (!ok) break;
                const int part = x.part, head0 = x.head0, row0 = x.row0;
                __syncwarp();
                mbar_arrive_if(lane == 0, bar(L::B_I_FREE + u % NI));
                if (!idle) {
                    const bool lost = l != l || top == INFINITY;  // NaN or an infinity among its scores: all NaN
                    const bool outgrown = !lost && (top > m + kGrowthLog2 || (fabsf(m) > kFarLog2 && m != -INFINITY));
                    const float by = l + up;
                    // a thread's row (of two groups: each half of the columns); rows with no weight (scale 0) become zeros whatever
                    // the columns hold
                    auto emit = [&](auto *to, float scale) {
                        using TOut = std::remove_pointer_t<decltype(to)>;
                        constexpr int E = 16 / (int)sizeof(TOut);
                        float found = 0.f;  // NaN where a value is not finite
                        to += D / NG * group;
#pragma unroll 1
                        for (int c0 = 0; c0 < D / NG; c0 += 32) {
                            float y[32];
                            tmem_ld32(t_o + D / NG * group + c0, y);  // (of no use where there is no tile)
#pragma unroll
                            for (int e = 0; e < 32; ++e) {
                                y[e] = scale == 0.f ? 0.f : y[e] * scale;
                                found = fmaf(y[e], 0.f, found);
                            }
                            if (valid) {
#pragma unroll
                                for (int e = 0; e < 32; e += E) store16<TOut>(to + c0 + e, y + e);
                            }
                        }
                        if (valid && (outgrown || (found != found && !lost))) {
                            const bool mark = outgrown || top > m + kSureLog2;
                            if (mark) *reinterpret_cast<uint2 *>(to) = make_uint2(kMarked, __float_as_uint(top));
                            say(mark && careful ? 2u | 16u : 1u);
                        }
                    };
                    if (part < 0) {
                        const int64_t row = row0 + tok;
                        if (group == 0 && valid && a.lse != nullptr) a.lse[(head0 + head) * a.q_total + row] = (m + log2f(l)) * kLn2;
                        emit(reinterpret_cast<__nv_bfloat16 *>(a.out) + (row * a.Hq + head0 + head) * D, lost ? NAN : l == 0.f ? 0.f : 1.f / by);
                    } else {
                        const int64_t at = (int64_t)part * a.part_rows + r;
                        if (group == 0 && valid) a.part_ml[at] = make_float4(m, l, by, 0.f);
                        emit(a.part_o + at * D, lost ? NAN : l == 0.f ? 0.f : 1.f);
                    }
                }
                tc_fence_before();  // (O has been read before the next P, or O_FREE, is announced)
                if (NG > 1 && n > 0) {
                    __syncwarp();
                    mbar_arrive_if(lane == 0, bar(L::B_O_FREE));
                }
            }
        };
        softmax(std::false_type{});
        if (another_pass()) {
            softmax(std::true_type{});
            another_pass();
            if ((wrong & 15u) == 11u) the_rest<D, kSoftmaxWarps>(a, run, smem, (wrong & 16u) != 0);  // (it takes far longer than a wait of another role may)
        }
    }
    if (warp == kScores) tmem_dealloc<1, L::COLS>(tmem);
}

// ---------------------------------------------------------------- host side
bool encode(CUtensorMap *m, const void *base, int rank, const cuuint64_t *dims, const cuuint64_t *strides, const cuuint32_t *box)
{
    auto fn = encode_fn();
    if (fn == nullptr) return false;
    const cuuint32_t ones[4] = {1, 1, 1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank, const_cast<void *>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// the query rows as (channel, head, token): a box is the heads of a block of as many tokens as a row tile holds
bool query_map(CUtensorMap *m, const PagedAttendArgs &a)
{
    const cuuint64_t dims[3] = {(cuuint64_t)a.c.D, (cuuint64_t)a.Hq, (cuuint64_t)a.q_total}, strides[2] = {(cuuint64_t)a.c.D * 2, (cuuint64_t)a.q_stride * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)a.block, (cuuint32_t)a.tokens};
    return encode(m, a.q, 3, dims, strides, box);
}
// a pool as (channel, slot, head, page): a box is a page's slots, or a tile's
bool pool_map(CUtensorMap *m, const PagedAttendArgs &a, const void *pool)
{
    const cuuint64_t dims[4] = {(cuuint64_t)a.c.D, (cuuint64_t)1 << a.c.page_log2, (cuuint64_t)a.c.Hkv, (cuuint64_t)a.c.n_pages},
                     strides[3] = {(cuuint64_t)a.c.slot_stride * 2, (cuuint64_t)a.c.head_stride * 2, (cuuint64_t)a.c.page_stride * 2};
    const cuuint32_t box[4] = {64, (cuuint32_t)a.box_rows, 1, 1};
    return encode(m, pool, 4, dims, strides, box);
}

template <int D>
cudaError_t launch(const PagedAttendArgs &a, const Maps &maps, cudaStream_t s)
{
    using L = Lay<D>;
    static Once once;
    const cudaError_t ready = once([] {
        cudaError_t e = cudaFuncSetAttribute(k_paged_tiles<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, L::BYTES);
        cudaFuncAttributes fa;
        if (e == cudaSuccess) e = cudaFuncGetAttributes(&fa, k_paged_tiles<D>);
        // (setmaxnreg would wait forever on registers that the launch does not have)
        return e != cudaSuccess ? e : (fa.numRegs + 7) / 8 * 8 < L::REGS ? cudaErrorInvalidConfiguration : cudaSuccess;
    });
    if (ready != cudaSuccess) return ready;
    return launch_chained(k_paged_tiles<D>, dim3((unsigned)a.runs), dim3(L::THREADS), L::BYTES, s, a, maps);
}

}  // namespace

cudaError_t launch_paged_tiles(PagedAttendArgs a, cudaStream_t s)
{
    a.box_rows = std::min(a.window == 0 ? BN : GR, 1 << a.c.page_log2);
    alignas(64) Maps maps;
    if (!query_map(&maps.q, a) || !pool_map(&maps.k, a, a.c.k) || !pool_map(&maps.v, a, a.c.v)) return cudaErrorInvalidValue;
    return a.c.D == 128 ? launch<128>(a, maps, s) : launch<64>(a, maps, s);
}

cudaError_t paged_tiles_error_words(unsigned int **wait, unsigned int **page)
{
    const cudaError_t e = cudaGetSymbolAddress(reinterpret_cast<void **>(wait), g_ris_paged_wait);
    return e != cudaSuccess ? e : cudaGetSymbolAddress(reinterpret_cast<void **>(page), g_ris_paged_page);
}

}  // namespace ris
