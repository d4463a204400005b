// Internal declarations of the serving operators: packed prompts, positions on several axes and
// the 4-bit cache (not part of the ABI).
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

#include "../../include/ris.h"
#include "once.h"
#include "ris_internal.h"

namespace ris {

constexpr int kPackRows = 128;      // query rows of a work item of a pack (one TMEM tile)
constexpr int kPackKeys = 128;      // keys of a key item
constexpr int kPackRuns = 304;      // runs of the keys of a long pack, about (two CTAs to an SM and head)
constexpr int kMaxAxes = 4;
constexpr int kCacheGroup = 32;     // elements that share a scale
constexpr int kMaxPackSeqs = 65535;
constexpr int kCacheUnit = 64;      // slots by which the attention over a 4-bit cache is shared out

// A work item: rows row .. row + kPackRows - 1 (or keys) of a sequence. The sequence's own sizes ride
// along, so that a CTA needs one 32-byte load to know everything about its item.
struct alignas(32) PackItem {
    int32_t seq;
    int32_t row;     // first row (or key) of the item within its sequence
    int32_t q_base;  // first row of the sequence in q / out
    int32_t q_len;
    int32_t k_base;  // first key of the sequence in k / v
    int32_t k_len;
    int32_t pad[2];
};

// A run of the keys of a sequence, by which the values are looked through and laid out.
struct alignas(32) PackRun {
    int32_t seq;
    int32_t first, n;    // its keys in k / v
    int32_t run0, run1;  // the runs of the sequence
    int32_t pad[3];
};

struct RopeAxesArgs {
    const void *x[2];          // q and k (k may be null: heads[1] = 0)
    void *y[2];
    int64_t stride[2];         // elements from one token's heads to the next's
    int32_t heads[2];
    int64_t n;
    int32_t D;
    const int32_t *pos;        // [axes][n]
    uint8_t axis[kMaxHeadDimHalf];   // axis of each frequency
    uint64_t turn[kMaxHeadDimHalf];  // rotation frequencies as fractions of a turn, in 2^-64
    float mscale;
    int32_t inverse;
};
cudaError_t launch_rope_axes(const RopeAxesArgs &a, int dtype, cudaStream_t s);

struct PackedArgs {
    const void *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;  // elements from token to token
    void *out;                 // [q_total][Hq][D]
    float *lse;                // [Hq][q_total] or null
    int64_t q_total, k_total;
    const PackItem *items;     // query items, the longest key range first
    int32_t n_items;
    const PackItem *key_items;
    int32_t n_key_items;
    int32_t Hq, Hkv, G;
    float scale_log2;          // log2(e) / sqrt(D)
    // key weights: of the last weight_rows rows of each sequence
    int32_t weight_rows;       // 0: none
    float *key_weight;         // [Hkv][k_total]
    float2 *row_stat;          // scratch [Hq][q_total]: each row's (maximum in log2, 1 / sum); null without weights
    const PackRun *runs;
    int32_t n_runs, n_seqs;
    uint8_t *far;              // tile kernels: [n_items][Hq][4] scratch, whose rows' scores passed what P's range allows
    const float *v_top;        // tile kernels: [n_seqs][Hkv] the largest |v|, or infinity where the rows are to be computed from
                               // the values as given (undefined for sequences without keys)
};
// fp32 inputs: items of kPackRows rows.
cudaError_t launch_packed_f32(const PackedArgs &a, int D, int out_dtype, cudaStream_t s);
cudaError_t launch_packed_weights_f32(const PackedArgs &a, int D, cudaStream_t s);
// bf16 inputs: items of kPackRows rows, or for clusters (head dim 128) with an odd group of 2 kPackRows;
// scratch of packed_scratch_bytes, 256-byte aligned.
size_t packed_scratch_bytes(const PackedArgs &a, int32_t head_dim);
cudaError_t launch_packed_tiles(PackedArgs a, int D, int out_dtype, bool clusters, void *scratch, cudaStream_t s);
cudaError_t launch_packed_weights_tc(const PackedArgs &a, int D, cudaStream_t s);

// Queries and keys normed per head and turned (norm_rope.cu): x into y, or backwards dy and x into y.
struct NormRopeArgs {
    const void *x[2];          // q and k (k may be null: heads[1] = 0)
    const void *dy[2];
    void *y[2];
    int64_t x_stride[2], dy_stride[2], y_stride[2];  // elements from one token's heads to the next's
    int32_t heads[2];
    int64_t n;
    const int32_t *pos;        // [n]
    const void *weight[2];     // [D] of the inputs' type; null: no norm
    float eps;
    int32_t rot;               // channels that are turned, a multiple of 16
    uint64_t turn[kMaxHeadDimHalf];  // rotation frequencies as fractions of a turn, in 2^-64
    float mscale;
    int32_t ctas[2];           // gradient: CTAs of q and of k
    float2 *part;              // [ctas[0] + ctas[1]][D] scratch, their sums for the weights (value, what is left of it)
};
cudaError_t launch_norm_rope(const NormRopeArgs &a, int dtype, int D, bool pairs, cudaStream_t s);
void norm_rope_ctas(int dtype, int D, int64_t n, const int32_t (&heads)[2], int32_t (&ctas)[2]);
cudaError_t launch_norm_rope_backward(const NormRopeArgs &a, int dtype, int D, bool pairs, float *gq, float *gk, cudaStream_t s);

// A cache in pages (paged.cu, attn_paged.cu).
struct PagedArgs {
    void *k, *v;               // pools of n_pages pages
    int64_t page_stride, head_stride, slot_stride;  // elements
    const int32_t *table;      // [B][table_len]
    int32_t *length;           // [B]
    int32_t B, Hkv, D, page_log2;
    int32_t n_pages, table_len;
};
struct PagedAppendArgs {
    PagedArgs c;
    const void *k, *v;
    int64_t k_stride, v_stride;
    const int32_t *start;      // [B] or null: the cache's lengths
    const int32_t *off, *seq_of;  // the pack's row offsets [B + 1] and sequence of each row
    int64_t total;
    int32_t rows;              // of a CTA
};
cudaError_t launch_paged_append(PagedAppendArgs a, int dtype, cudaStream_t s);

// A row tile's part that a run leaves for the join: parts of runs first .. last, -1: none.
struct PagedSplit {
    int32_t first, last;
    int32_t row0, tokens;      // its first row in q / out, its tokens
    int32_t head0, heads;      // its query heads
    int32_t pad[2];
};
struct PagedItem {
    int32_t seq, tile;
};
struct PagedAttendArgs {
    PagedArgs c;
    const void *q;
    void *out;                 // [q_total][Hq][D]
    float *lse;                // [Hq][q_total] or null
    int64_t q_stride, q_total;
    const int32_t *off;        // the pack's row offsets [B + 1]
    int32_t Hq, G;
    int32_t block, blocks;     // query heads of a row tile; how many such blocks a KV head has
    int32_t tokens;            // of a row tile
    int32_t window, anchors;   // window 0: all
    int32_t reach;             // lengths count up to here
    float scale_log2;
    int32_t box_rows;          // tile kernel: keys of a TMA box
    int64_t wait_limit;        // tile kernel: cycles that a wait may take
    int32_t debug_no_loads;    // tile kernel, tests only: no copies are issued, so the first wait on them gives up
    // the sharing out of the work (attn_paged.cuh)
    int64_t line;              // row tiles of the line (at most)
    int32_t unit_cost;         // what a row tile costs besides its key tiles
    int32_t runs;              // of the line, one for each CTA
    int32_t max_items;         // 0: a row tile per sequence, else as many items as the plan has room for
    int64_t *prefix;           // [max_items + 1] scratch: cost of the items before
    PagedItem *items;          // [max_items]
    int32_t *n_items;          // [1]
    int32_t *seq_items;        // [B] first item of each sequence
    PagedSplit *split;         // [runs]
    int32_t part_rows;         // rows of a part
    float *part_o;             // [2 runs][part_rows][D]
    float4 *part_ml;           // [2 runs][part_rows] (reference in log2, sum, what the outputs are divided by)
};
constexpr int kPagedSMs = 152;
// keys of a key tile and rows of a row tile, fp32 (by the most rows that a sequence has) and bf16
constexpr int kPagedF32Keys = 64, kPagedTileRows = 128, kPagedTileKeys = 128, kPagedGranule = 32;
int32_t paged_f32_rows(int64_t rows);
// in key tiles, what a row tile costs besides them
constexpr int paged_unit_cost(bool tiles, int D) { return !tiles ? 1 : D == 128 ? 5 : 3; }
constexpr int paged_tile_ctas(int D) { return D == 128 ? 1 : 2; }
cudaError_t launch_paged_plan(const PagedAttendArgs &a, int dtype, cudaStream_t s);
cudaError_t launch_paged_join(const PagedAttendArgs &a, int dtype, cudaStream_t s);
cudaError_t launch_paged_f32(const PagedAttendArgs &a, int32_t rows, cudaStream_t s);
cudaError_t launch_paged_tiles(PagedAttendArgs a, cudaStream_t s);

struct Cache4Args {
    uint8_t *k, *v;              // [B][Hkv][cap][D / 2]
    uint16_t *k_scale, *v_scale; // bf16 [B][Hkv][cap][D / 32]
    int32_t *pos;                // [B][Hkv][cap]
    float *weight;               // [B][Hkv][cap]
    int32_t *length;             // [B]
    int32_t B, Hkv, D;
    int64_t cap;
};

struct Cache4AppendArgs {
    Cache4Args c;
    const void *k, *v;
    int64_t k_stride, v_stride;
    const int32_t *positions;    // [total]
    const float *weight;         // [Hkv][total] or null (zero)
    const int32_t *start;        // [B] or null: the cache's lengths
    const int32_t *off;          // the pack's row offsets [B + 1]
    const int32_t *seq_of;       // sequence of each row [total]
    int64_t total;
    unsigned int *ticket;        // start null: CTAs done (0 between calls)
};
cudaError_t launch_cache4_append(const Cache4AppendArgs &a, int dtype, cudaStream_t s);
// The lengths of an append without rows.
cudaError_t launch_cache4_start(const Cache4Args &c, const int32_t *start, cudaStream_t s);
cudaError_t launch_cache4_read(const Cache4Args &c, const int32_t *first, int64_t count, float *k, float *v, cudaStream_t s);

struct Cache4AttendArgs {
    Cache4Args c;
    const void *q;               // [B][Hq][D]
    void *out;
    float *lse;                  // [B][Hq] or null
    const float *weight_in;      // [B][Hkv][cap] or null
    float *weight_out;           // or null
    int32_t Hq, G;
    float scale_log2;
    int64_t reach;               // slots that a sequence can hold: cap, or less where the caller knows better
    int32_t lists;               // (sequence, KV head, block of 8 query heads)
    int32_t ctas;                // among which the slots are shared out
    float *part_o;               // [ctas + lists][heads of a block][D]
    float2 *part_ml;             // [ctas + lists][heads of a block]
    int32_t *list_cta;           // [lists][2] first and last CTA of each list that holds slots
    float *scores;               // weights: [B][Hq][score_pitch] scores in log2
    int64_t score_pitch;         // reach, rounded up to a multiple of 4
    int64_t wait_limit;          // cycles a device-side wait may take (0: about 2^31)
    int32_t debug_no_loads;      // tests only: no copies are issued, so the first wait on them gives up
};
cudaError_t launch_cache4_attend(Cache4AttendArgs a, int dtype, int out_dtype, cudaStream_t s);

struct Cache4EvictArgs {
    Cache4Args src, dst;
    int32_t in_place;
    int32_t budget, recent;
    int32_t *kept;               // [B][Hkv][budget]
};
// holes: scratch [B * Hkv][budget]
cudaError_t launch_cache4_evict(const Cache4EvictArgs &a, int32_t *holes, cudaStream_t s);

// The device error words of the cache's kernels (bit 1: tokens appended past the capacity, bit 2: a bounded
// wait gave up) and of the packed attention's tile kernels (a bounded wait gave up), on the current device.
cudaError_t cache4_error_word(unsigned int **p);
cudaError_t packed_error_word(unsigned int **p);
// Of the paged cache's kernels: a token or key outside the pages; of its tile kernel alone: a bounded wait gave
// up, a key outside the pages.
cudaError_t paged_error_word(unsigned int **p);
cudaError_t paged_tiles_error_words(unsigned int **wait, unsigned int **page);

// What ris_debug_tile_stall asks for (ris_api.cu): cycles that a wait may take, 0 where nothing is asked;
// whether loads are left out.
int64_t debug_wait_limit();
int32_t debug_no_loads();

// Stream-ordered pool memory, as every allocation of the library (ris_api.cu).
cudaError_t library_alloc(void **p, size_t bytes, cudaStream_t s);

#ifdef __CUDACC__
// The serving kernels are a few microseconds each, one after another: each is launched while the last one
// runs (a programmatic dependent) and waits for it where it begins, so that only the launch itself
// overlaps: nothing is read or written before `after_last` returns. Its own dependent may start from there
// on.
__device__ __forceinline__ void after_last()
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}
template <typename... P, typename... A>
cudaError_t launch_chained(void (*kern)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t s, const A &...args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kern, P(args)...);
    note_launch();
    return e != cudaSuccess ? e : cudaGetLastError();
}
#endif

}  // namespace ris
