/*
 * ris.h -- C ABI of libris, the GB300 (sm_103a) implementation of RIS (Reduced
 * Interaction Sampling) prefill sparse self-attention, arxiv 2607.21927.
 *
 * Conventions shared by every call
 *   - Tensors are caller-owned, contiguous, token-major DEVICE pointers unless a comment
 *     says "host". q is [N][heads][head_dim], k and v are [N][kv_heads][head_dim], out is
 *     [N][heads][head_dim] (per-seed calls: [n_seeds][N][heads][head_dim]).
 *     Every device pointer must be 16-byte aligned.
 *   - `stream` is a cudaStream_t passed as void* (NULL = the legacy default stream). Calls
 *     are stream-ordered and asynchronous unless their comment says "blocks".
 *   - Each call returns a ris_status. Arguments are validated before anything is launched;
 *     an invalid call launches nothing and returns RIS_ERR_INVALID. The text of the last
 *     error of the calling thread is returned by ris_last_error(). A device fault of an
 *     earlier launch surfaces as RIS_ERR_CUDA from a later call or at the caller's sync.
 *   - There is no CPU fallback: without a CUDA device every compute call returns
 *     RIS_ERR_CUDA.
 *   - Temporary device memory is taken from the device's stream-ordered pool
 *     (cudaMallocAsync on `stream`) and released on the same stream.
 */
#ifndef RIS_H
#define RIS_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    RIS_OK = 0,
    RIS_ERR_INVALID = 1,        /* bad argument; nothing was launched */
    RIS_ERR_OOM = 2,            /* device allocation failed */
    RIS_ERR_CUDA = 3,           /* a CUDA runtime call failed (or no device) */
    RIS_ERR_UNSUPPORTED = 4,    /* valid but not built (e.g. head_dim outside {64,128}) */
    RIS_ERR_DEVICE_TIMEOUT = 5  /* a bounded device-side wait gave up */
} ris_status;

/* Sampling modes (paper, Methods, "Sampling Modes: Stochastic and Structural"). */
typedef enum {
    RIS_MODE_STOCHASTIC = 0, /* the whole density budget drawn uniformly per pivot row */
    RIS_MODE_STRUCTURAL = 1, /* block cliques of B = min(0.1 N, round(d N)) + global draws */
    RIS_MODE_DENSE = 2       /* every causal pair (the dense upper bound, Table tab:results_32k) */
} ris_mode;

typedef enum { RIS_F32 = 0, RIS_BF16 = 1 } ris_dtype;

/* RoPE position extension (Methods, "Dynamic RoPE Scaling"). */
typedef enum { RIS_ROPE_NONE = 0, RIS_ROPE_PLAIN = 1, RIS_ROPE_LINEAR = 2, RIS_ROPE_YARN = 3 } ris_rope_kind;

typedef struct {
    int32_t kind;       /* ris_rope_kind */
    int32_t reserved;   /* must be 0 */
    double theta;       /* base, e.g. 1e6 (Qwen2) or 1e4 (TinyLlama) */
    int64_t native_len; /* trained positional limit, e.g. 32768 or 2048 */
    double factor;      /* extension factor s; <= 0 resolves to max(1, N / native_len) */
    double yarn_alpha;  /* YaRN ramp start in rotations per native window (default 1) */
    double yarn_beta;   /* YaRN ramp end (default 32) */
} ris_rope_cfg;

/* Forced set and keying of a mask; NULL means all defaults. */
typedef struct {
    int32_t local_window; /* W >= 1: keys i-W < j <= i always kept (1 = diagonal only, default) */
    int32_t n_anchor;     /* A >= 0: keys j < A always kept (global anchors, default 0) */
    int32_t per_head;     /* 0: one mask shared by all heads (default); 1: one mask per KV head */
    uint32_t layer_key;   /* mixed into every draw; 0 = shared across layers (default) */
    int32_t sampler;      /* random part: 0 = Bernoulli keep test per causal pair (default);
                             1 = index draws: per row and seed, `draws` indices j drawn with
                             replacement uniformly over [0, N), kept when j < i, repeats merged
                             (the torch.randint wording of Methods, "Memory-Bounded Geometry
                             Generation") */
} ris_mask_opts;

/* The paper's three-part geometry (Results, "Ensemble Stochastic Projection and Retrieval
 * Coverage"): a dense local window of 1024 tokens, a global anchor over the initial tokens
 * and the stochastic ensemble. The paper does not give the anchor count; 4 initial tokens
 * (the attention-sink count of streaming attention) is this library's reading. Use as
 * ris_mask_opts{RIS_PRESET_LOCAL_WINDOW, RIS_PRESET_ANCHORS, 0, 0, 0}. */
#define RIS_PRESET_LOCAL_WINDOW 1024
#define RIS_PRESET_ANCHORS 4

/* Derived scalars of one call, resolved on the host. */
typedef struct {
    int64_t bmax;            /* K = floor(d N + 0.5), the paper's B_max */
    int64_t block;           /* Structural block size B = max(1, min(floor(N/10), K)) */
    int64_t clique_pairs;    /* C, causal clique pairs of all blocks */
    double d_clique;         /* C / N^2 */
    double d_global;         /* max(0, d - d_clique): Structural global draw density */
    uint64_t thr;            /* keep iff Philox word < thr; 2^32 = always */
    uint32_t stream;         /* Philox counter word 2: 0 Stochastic draws, 1 Structural global */
    int32_t dense;           /* 1 when every causal pair is kept (dense mode or density 1) */
    double rope_factor;      /* resolved s */
    double rope_mscale;      /* 0.1 ln s + 1 for YaRN, else 1 */
    int64_t draws;           /* index-draw sampler: draws per row and seed, floor(d N + 0.5) for
                                Stochastic, floor(d_global N + 0.5) for Structural */
} ris_params;

/* Opaque handle to a mask held in device memory. */
typedef struct ris_mask_s *ris_mask_t;

/* Device-side layout of a mask, read by ris_mask_info. All pointers are owned by the mask.
 *   n_masks = (per_seed ? n_seeds : 1) * (per_head ? kv_heads : 1); mask m = s * heads_keyed + h.
 *   CSR: keys of row i of mask m are col[row_ptr[m*N + i] .. row_ptr[m*N + i + 1]),
 *        ascending, int64 row_ptr of n_masks*N + 1 entries, col of col_bytes (2 if N <= 65536,
 *        else 4) each.
 *   Bitmap: row i of mask m holds words floor(i/32)+1 words at
 *        bitmap + m * words_per_mask + row_word_offset(i), with
 *        row_word_offset(32a + b) = 32a + b + 16 a (a - 1) + a b; bit (j mod 32) of word j/32
 *        is pair (i, j); bits above the diagonal are zero.
 *   Dense masks (mode DENSE or density 1) store nothing: row_ptr, col and bitmap are NULL
 *   and row i holds keys 0..i. */
typedef struct {
    int64_t N;
    int32_t n_masks;
    int32_t heads_keyed;   /* 1, or kv_heads when per_head */
    int32_t n_seeds;
    int32_t per_seed;
    int32_t col_bytes;
    int32_t dense;
    int64_t n_pairs;       /* total stored pairs over all masks */
    int64_t words_per_mask;
    const int64_t *row_ptr;
    const void *col;
    const uint32_t *bitmap;
    ris_params params;
    int64_t suffix_pairs;  /* pairs per mask in the rows' dense suffixes: keys lo(i) .. i of row i,
                              all kept, lo(i) the earlier of the row's Structural block start
                              (blocks of >= 256 tokens) and its local window start (0 when the
                              mask is dense, per seed, or has neither span of >= 256); the
                              dense-suffix split attends these on the tiles */
} ris_mask_desc;

/* Resolve the scalars of a call on the host (no device work, usable without a GPU).
 * Structural geometry follows Methods, "Sampling Modes"; B_max = round(d N) matches the
 * B_max column of the sub-1% sweet-spot table. rope may be NULL (factor 1, mscale 1).
 * Returns RIS_ERR_INVALID for N < 1, density outside (0, 1], an unknown mode or rope kind. */
ris_status ris_resolve_params(int64_t N, int32_t mode, double density, const ris_rope_cfg *rope,
                              ris_params *out);

/* RoPE rotation frequencies f[head_dim/2] (host array, fp64) and the vector scale for a
 * sequence of N tokens: plain theta^(-2k/D); linear f/s; YaRN ramp between the two
 * (Methods, "Dynamic RoPE Scaling"; YaRN per Peng et al. 2023). No device work. */
ris_status ris_rope_freqs(const ris_rope_cfg *rope, int64_t N, int32_t head_dim, double *f_out,
                          double *mscale_out);

/* Build the RIS mask of N tokens (Methods, "Memory-Bounded Geometry Generation" and
 * "Sampling Modes"): for every seed, keep causal pair (i, j<i) iff Philox4x32-10 word
 * (j mod 4) of key (seed, head_key) and counter (j/4, i, stream, layer_key) is below thr
 * (opts->sampler 0), or (sampler 1) iff j < i is one of the row's `draws` indices
 * j_t = floor(u_t N / 2^32), u_t word (t mod 4) of key (seed, head_key) and counter
 * (t/4, i, stream + 2, layer_key);
 * Structural adds the block cliques; the forced local window and anchors are added; with
 * per_seed = 0 all seeds are OR-merged into one master mask, with per_seed = 1 each seed
 * keeps its own mask. Output: bitmap + CSR in device memory owned by *out_mask.
 * seeds: HOST array of n_seeds values, 1 <= n_seeds <= 256. kv_heads is used only when
 * opts->per_head = 1. Blocks: the CSR size is read back before the key lists are written.
 * The wait covers `stream` only: a mask built on a stream of its own (ordered before the
 * attention calls that read it, and freed after them) leaves work queued on other streams
 * running while the host waits.
 * Errors: RIS_ERR_INVALID (N < 1 or > 2^31, density outside (0,1], bad opts or seeds),
 * RIS_ERR_OOM, RIS_ERR_CUDA. On error *out_mask is NULL. */
ris_status ris_mask_generate(int64_t N, int32_t kv_heads, int32_t mode, double density,
                             const uint32_t *seeds, int32_t n_seeds, const ris_mask_opts *opts,
                             int32_t per_seed, ris_mask_t *out_mask, void *stream);

/* Describe a mask (host struct filled from host-side metadata; no device work). */
ris_status ris_mask_info(ris_mask_t mask, ris_mask_desc *out);

/* Release a mask's device memory, ordered on the stream it was built on. NULL is a no-op. */
ris_status ris_mask_free(ris_mask_t mask);

/* Rotate x[N][heads][head_dim] in place with RoPE (rotate-half pairs (c, c + D/2)) at
 * positions 0..N-1, then scale by mscale (Methods, "Dynamic RoPE Scaling"). Angles are
 * formed and reduced in fp64; the rotation runs in fp32; bf16 results are rounded to
 * nearest even. head_dim must be even. Errors: RIS_ERR_INVALID. */
ris_status ris_rope_apply(void *x, int32_t dtype, int64_t N, int32_t heads, int32_t head_dim,
                          const ris_rope_cfg *rope, void *stream);

/* RIS sparse attention of one layer (Methods, "Hybrid Anchor and Pre-Fusion Unified Softmax"):
 *   out[i][h] = sum_{j in M_i} softmax_j(<q~_i,h , k~_j,g> / sqrt(D)) v_j,g,  g = h / (heads/kv_heads)
 * with one softmax over the whole key set M_i of the master mask (all seeds OR-merged), q~ and
 * k~ rotated by `rope` (NULL or kind NONE: q and k are used as given). Builds the mask, runs
 * the attention and frees the mask, all on `stream`; blocks once while the mask is sized, unless the
 * key lists of every causal pair would fit in 64 MiB (about N = 8190). Such a call does not know the
 * mask's pair count and chooses its design (see ris_attention_design) from the expected one: near the
 * line between two designs it may take the other than ris_attention_masked on the built mask, with
 * outputs that differ in their last bits.
 * dtype: q, k, v element type; out_dtype: out element type (F32 or BF16). lse: optional
 * [heads][N] fp32 natural-log sum of exp of the scaled scores (NULL to skip).
 * head_dim in {64, 128}; heads a multiple of kv_heads; heads/kv_heads <= 8, or any group size
 * with bf16 inputs, which then always run on the tile design (the gathers carry at most 8
 * query heads per KV head; otherwise RIS_ERR_UNSUPPORTED; the decode step keeps the limit
 * of 8).
 * Errors: RIS_ERR_INVALID, RIS_ERR_UNSUPPORTED, RIS_ERR_OOM, RIS_ERR_CUDA. */
ris_status ris_sparse_attention_fwd(const void *q, const void *k, const void *v, void *out,
                                    int64_t N, int32_t heads, int32_t kv_heads, int32_t head_dim,
                                    int32_t mode, double density, const uint32_t *seeds,
                                    int32_t n_seeds, int32_t dtype, int32_t out_dtype,
                                    const ris_rope_cfg *rope, const ris_mask_opts *opts, float *lse,
                                    void *stream);

/* The attention step alone on a mask built by ris_mask_generate (the mask is built once per
 * prefill and reused by every layer, Methods, "Memory-Bounded Geometry Generation"). With a
 * per-seed mask, out is [n_seeds][N][heads][head_dim] and lse [n_seeds][heads][N].
 * kv_heads must equal the mask's kv_heads when it is keyed per head. Asynchronous.
 * Errors: as ris_sparse_attention_fwd. */
ris_status ris_attention_masked(ris_mask_t mask, const void *q, const void *k, const void *v,
                                void *out, int32_t heads, int32_t kv_heads, int32_t head_dim,
                                int32_t dtype, int32_t out_dtype, const ris_rope_cfg *rope,
                                float *lse, void *stream);

/* Ensemble of per-seed sparse views in one launch: seed s attends over F + M_s only and
 * writes out[s] (the "independent sparse views" read of Results, "Linear Interpolation";
 * union coverage of Eq. union_coverage is the OR of these views). Same arguments as
 * ris_sparse_attention_fwd; out is [n_seeds][N][heads][head_dim], lse [n_seeds][heads][N]. */
ris_status ris_ensemble_batch(const void *q, const void *k, const void *v, void *out, int64_t N,
                              int32_t heads, int32_t kv_heads, int32_t head_dim, int32_t mode,
                              double density, const uint32_t *seeds, int32_t n_seeds,
                              int32_t dtype, int32_t out_dtype, const ris_rope_cfg *rope,
                              const ris_mask_opts *opts, float *lse, void *stream);

/* Query rows row_begin .. row_end-1 of ris_attention_masked (same arguments otherwise): the
 * other rows of out and lse are left untouched, and each computed row equals the same row of
 * the whole-layer call bit for bit. K and V must still hold every position (any row may
 * attend to any earlier key). This is how one prefill is split across devices or streams:
 * query rows are independent given K, V and the counter-based mask (each device can build the
 * same mask), so each part needs no exchange. Errors: as ris_attention_masked, and
 * RIS_ERR_INVALID for an empty range or one outside [0, N). */
ris_status ris_attention_masked_rows(ris_mask_t mask, int64_t row_begin, int64_t row_end, const void *q,
                                     const void *k, const void *v, void *out, int32_t heads, int32_t kv_heads,
                                     int32_t head_dim, int32_t dtype, int32_t out_dtype, const ris_rope_cfg *rope,
                                     float *lse, void *stream);

/* Query rows row_begin .. row_end-1 of ris_attention_masked with only those rows in memory:
 * q_rows [row_end - row_begin][heads][head_dim] holds query rows row_begin .., out_rows gets
 * the same rows of the output, and lse_rows (optional) is [heads][row_end - row_begin]. K and V
 * must hold every position 0 .. N-1: this is the per-device step of a prefill split by query
 * rows in which each device holds only its own rows of q, k and v and all-gathers the layer's
 * K and V first (the paper's row independence, Methods, "Memory-Bounded Geometry Generation":
 * every device builds the same counter-based mask). Each row equals the same row of the
 * whole-layer call bit for bit, except that with rotated bf16 inputs at head dim 128 the power-of-two
 * scales of the score operands follow from the largest pair norm (elements c and c + 64) of the queries
 * given: where the whole layer's is in another binade, last bits may differ. Masks built per seed are refused (RIS_ERR_UNSUPPORTED).
 * Errors: as ris_attention_masked_rows. */
ris_status ris_attention_masked_local(ris_mask_t mask, int64_t row_begin, int64_t row_end, const void *q_rows,
                                      const void *k, const void *v, void *out_rows, int32_t heads, int32_t kv_heads,
                                      int32_t head_dim, int32_t dtype, int32_t out_dtype, const ris_rope_cfg *rope,
                                      float *lse_rows, void *stream);

/* Balanced contiguous row ranges for `parts` workers: bounds[0] = 0 < bounds[1] < ... <
 * bounds[parts] = N, cut where the running sampled-pair count reaches k/parts of the total
 * (every part gets at least one row). ris_row_split takes a HOST row_ptr of N + 1 offsets
 * (no device work); ris_mask_row_split reads the mask's own counts (summed over its per-seed
 * or per-head masks; row i of a dense mask counts i + 1) and blocks. Errors: RIS_ERR_INVALID
 * (NULL, parts outside [1, N]), RIS_ERR_CUDA. */
ris_status ris_row_split(const int64_t *row_ptr, int64_t N, int32_t parts, int64_t *bounds);
ris_status ris_mask_row_split(ris_mask_t mask, int32_t parts, int64_t *bounds);

/* Allocation-free variant of ris_attention_masked: same arguments and the same results
 * within the parity tolerance (not bit for bit), with these differences.
 * The paper has no counterpart: this entry point exists for callers that may not allocate
 * device memory while a layer runs, such as an inference engine's enqueue callback that may
 * only launch work, or a server that plans all device memory at load time. They build the
 * mask once beforehand (ris_mask_generate allocates) and call this per layer.
 *   - Every mask runs on the register gather (fp32: the fp32 gather), whatever design
 *     ris_attention_masked would pick: dense and high-density masks run at gather speed, not
 *     on the tiles, and heads / kv_heads above 8 are refused (RIS_ERR_UNSUPPORTED).
 *   - Instead of the stream-ordered pool, the rotated q (fp32) and k (bf16 hi + lo, or fp32)
 *     live in one library-owned device array of 64 MiB per device. Every GPU on which the
 *     library's device code is loaded holds it until the process exits: with lazy module
 *     loading (the CUDA default) the GPUs on which a kernel of this library ran, with
 *     CUDA_MODULE_LOADING=EAGER every context that loads the library. The call needs
 *       align256(N*heads*head_dim*4) + (bf16 ? 2 : 1) * align256(N*kv_heads*head_dim*(bf16 ? 2 : 4))
 *     bytes when rope is set (none without rope) and returns RIS_ERR_INVALID, launching
 *     nothing, when that exceeds 64 MiB (about N = 9300 tokens at 12 / 2 heads of 128).
 * It calls no allocation routine. The first call in a device's context looks up the array's
 * device address (and may load the library's device code): make that first call before any
 * stream capture; a context created anew (after cudaDeviceReset) is looked up again.
 * Every call on a device shares the array and leaves its contents behind; each call writes
 * all scratch it reads, so nothing needs clearing, but calls whose GPU work overlaps (e.g.
 * on two streams) race on it and must be ordered by the caller. */
ris_status ris_attention_masked_noalloc(ris_mask_t mask, const void *q, const void *k, const void *v,
                                        void *out, int32_t heads, int32_t kv_heads, int32_t head_dim,
                                        int32_t dtype, int32_t out_dtype, const ris_rope_cfg *rope,
                                        float *lse, void *stream);

/* The allocation-free entry point's scratch array in the current device's context: its
 * device address and size in bytes (the paper has no counterpart). Looks the address up like
 * the entry point's first call does. Errors: RIS_ERR_INVALID (NULL outputs), RIS_ERR_CUDA. */
ris_status ris_noalloc_scratch_info(void **device_address, int64_t *bytes);

/* Kernel timer for measurement (off by default). While enabled, every attention kernel launch
 * (the fused QK^T -> softmax -> PV kernel of a layer, or a decode step's two kernels; not
 * RoPE or mask kernels) is bracketed by CUDA events recorded on the stream it is launched on. Enabling or
 * disabling clears the record.
 * ris_kernel_timer_read blocks until the last recorded launch has finished, returns the summed
 * device milliseconds and the number of launches recorded since the last read, and clears
 * them. Intended for one thread at a time. Errors: RIS_ERR_INVALID (NULL outputs), RIS_ERR_CUDA. */
ris_status ris_kernel_timer_enable(int32_t enable);
ris_status ris_kernel_timer_read(double *total_ms, int64_t *launches);
/* As ris_kernel_timer_read, and also the duration of each of the first `capacity` recorded
 * launches, in launch order, into the HOST array ms_each (NULL when capacity is 0). */
ris_status ris_kernel_timer_samples(double *total_ms, int64_t *launches, double *ms_each, int64_t capacity);

/* Attention kernel design a layer call on `mask` uses for this input dtype and head_dim
 * (host-only, no device work): 0 register gather, 2 tcgen05 masked dense tiles,
 * 3 fp32 gather, 4 dense-suffix split; -1 for invalid arguments. bf16 calls use tiles when
 * the mask is dense or keeps at least 5.8% (head_dim 128) or 8.8% (head_dim 64) of the
 * causal pairs (up to 2.25 times that below 3072 tokens) in what a gather would fetch (and
 * always when heads/kv_heads > 8, which this call does not see). The dense-suffix split applies to
 * masks (not per seed) with Structural blocks of at least 256 tokens or a local window of at least 256 keys: every key of row i
 * from the earlier of its block start and its window start up to i is kept (Methods,
 * "Sampling Modes": in-block pairs are cliques; the window is forced), so a first launch
 * attends every row to that suffix on the tiles and the register gather continues that
 * softmax over the row's other keys; the result is the same single softmax over the row's
 * whole key set. RIS_FORCE_DESIGN = gather | tile | suffix in the environment
 * overrides (benchmarking). */
int32_t ris_attention_design(ris_mask_t mask, int32_t dtype, int32_t head_dim);

/* Synchronise `stream` and report (then clear) the device error words: RIS_ERR_DEVICE_TIMEOUT
 * if a kernel's bounded wait gave up since the last call, RIS_ERR_INVALID if a decode step
 * read a position outside [t0, cache_len) from device memory, tokens did not fit a 4-bit cache, or tokens or keys
 * lie outside a cache's pages, else RIS_OK. A kernel that sets
 * a word skips the rest of its work, so outputs of that launch are undefined. Blocks.
 * Errors: RIS_ERR_CUDA. */
ris_status ris_device_status(void *stream);

/* Release the library's cached per-device state (the paper has no counterpart): the kernel
 * timer's events, and the device memory that the stream-ordered pools of the devices this
 * library used keep cached (each pool is trimmed and its release threshold set back to the
 * CUDA default, 0). The allocation-free entry point's scratch array is a static device
 * array: it stays mapped until the process exits, and its address is looked up again on the
 * next call. Live masks and anchors stay valid and are still released by ris_mask_free /
 * ris_anchor_free. Testing switches (ris_debug_*) are reset. The library may be used again
 * afterwards. Call it with no library work in flight on any stream. Errors: RIS_ERR_CUDA. */
ris_status ris_shutdown(void);

/* ---- Failure injection for tests (the paper has no counterpart) ---------------------------
 * ris_debug_fail_allocation: the n-th stream-ordered device allocation the library makes from
 * now on (0 = the next one) fails as if the pool were exhausted; later ones succeed again.
 * n < 0 disarms. Every entry point must then return RIS_ERR_OOM, leave its output handle NULL
 * and release, on its stream, whatever it had allocated.
 * ris_debug_tile_stall: with no_loads = 1 the tile kernel's loader issues no copies, so its
 * first wait on them gives up after wait_limit_cycles (0 = the default, about 2^31 cycles):
 * the kernel sets its device error word, releases its tensor memory and returns, and
 * ris_device_status reports RIS_ERR_DEVICE_TIMEOUT (outputs of that launch are undefined).
 * The copies of ris_cache4_attend and, in bf16, of ris_paged_attend are left out and waited for in the same way.
 * no_loads = 0 with a nonzero limit only shortens the waits. (0, 0) restores the defaults.
 * Both switches are process-wide. Errors: RIS_ERR_INVALID. */
ris_status ris_debug_fail_allocation(int64_t n);
ris_status ris_debug_tile_stall(int32_t no_loads, int64_t wait_limit_cycles);

/* ---- Hybrid Anchor decode (Methods, "Hybrid Anchor and Pre-Fusion Unified Softmax (PFUS)") ----
 * After a prefill of n_prefill tokens, the token generated at position t >= t0 = n_prefill
 * attends, with one softmax, to the union of
 *   - the Stochastic Anchor: the key set of the first generated token, computed once and frozen.
 *     It is row t0 of the prefill's RIS mask (same mode, density, seeds, anchors n_anchor,
 *     per_head / layer_key keying and sampler; parameters resolved for n_prefill tokens)
 *     without its local window: every kept key j < t0;
 *   - the Dynamic Local Window: keys t - window < j <= t.
 * Duplicates are merged (each key counts once). The K/V cache holds the rotated keys. */
typedef struct ris_anchor_s *ris_anchor_t;

/* Build the Stochastic Anchor on the device (one mask row per KV head when opts->per_head,
 * else one) and keep a host copy of its keys for the per-step merge. opts->local_window is
 * ignored (the decode step has its own window). Blocks (reads the key count back).
 * Errors: as ris_mask_generate; RIS_ERR_INVALID also for n_prefill >= 2^31 - 1. */
ris_status ris_decode_anchor(int64_t n_prefill, int32_t kv_heads, int32_t mode, double density,
                             const uint32_t *seeds, int32_t n_seeds, const ris_mask_opts *opts,
                             ris_anchor_t *out, void *stream);

/* Layout of an anchor: t0, number of keyed lists (1 or kv_heads), total keys, and DEVICE
 * pointers to the keys (int32, ascending within each list) and the heads_keyed + 1 int64
 * offsets (list m = keys[offsets[m] .. offsets[m+1])). Any output pointer may be NULL. */
ris_status ris_anchor_info(ris_anchor_t anchor, int64_t *t0, int32_t *heads_keyed, int64_t *n_keys,
                           const int32_t **keys, const int64_t **offsets);
ris_status ris_anchor_free(ris_anchor_t anchor);

/* Rotate x [n][heads][head_dim] (dtype) at positions pos0 .. pos0+n-1 into hi (same dtype)
 * and, for bf16 when lo is not NULL, lo = bf16(y - bf16(y)) so that hi + lo carries the fp32
 * rotation to ~16 bits: the format of a rotated K cache. The extension factor is resolved
 * for n_ctx tokens (rope->factor <= 0). rope NULL or RIS_ROPE_NONE copies x (no rotation).
 * x and hi may be the same buffer. Errors: RIS_ERR_INVALID, RIS_ERR_CUDA. */
ris_status ris_rope_split(const void *x, int32_t dtype, int64_t n, int64_t pos0, int32_t heads, int32_t head_dim,
                          int64_t n_ctx, const ris_rope_cfg *rope, void *hi, void *lo, void *stream);

/* One decode step. q: [heads][head_dim] query of the token at position t, NOT rotated (the
 * kernel rotates it at position t with the extension factor of n_ctx tokens). k (+ k_lo for
 * bf16, may be NULL) and v: the cache [cache_len][kv_heads][head_dim] holding positions
 * 0 .. cache_len-1 with rotated keys (ris_rope_split); it must already hold the token t's own
 * key and value. out: [heads][head_dim] (out_dtype); lse: [heads] natural-log sum of
 * exp(score) or NULL. Scores and probabilities are fp32.
 * Position: t (host value) when t_dev is NULL; otherwise the int64 at t_dev (device memory,
 * 8-byte aligned) is read when the step runs and t is ignored, and with advance != 0 the
 * step adds 1 to *t_dev when it has finished. Nothing in the launch then depends on the
 * position, so a captured CUDA graph of a token's steps can be replayed token after token.
 * A device-side position outside [t0, cache_len) makes the step attend to nothing (undefined
 * output) and is reported by ris_device_status as RIS_ERR_INVALID.
 * Partial results live in a buffer owned by the anchor, grown by the first call of a larger
 * shape (stream-ordered pool allocation: make that call before any stream capture); steps on
 * one anchor must therefore be ordered on the GPU (one stream, or events between streams).
 * Errors: RIS_ERR_INVALID (host t outside [t0, cache_len), window < 1, shapes, pointers,
 * anchor keyed for another kv_heads, advance without t_dev), RIS_ERR_UNSUPPORTED
 * (kv_heads > 64), RIS_ERR_CUDA. */
ris_status ris_decode_step(ris_anchor_t anchor, const void *q, const void *k, const void *k_lo, const void *v,
                           int64_t cache_len, int64_t t, int64_t *t_dev, int32_t advance, int32_t window,
                           int32_t heads, int32_t kv_heads, int32_t head_dim, int32_t dtype, int32_t out_dtype,
                           int64_t n_ctx, const ris_rope_cfg *rope, void *out, float *lse, void *stream);

/* ---- Packed prompts and a 4-bit cache ---------------------------------------------------------
 * The serving path of a batch of sequences (the paper has no counterpart): positions given per
 * token, causal attention over prompts of different lengths in one call, a K/V cache held in 4
 * bits, and its eviction by accumulated attention weight.
 *
 * Pack: the plan of a call over n_seqs sequences whose tokens lie one after another. Sequence s has
 * q_lens[s] rows (new tokens) and k_lens[s] keys (HOST arrays; k_lens NULL: the same lengths). The rows
 * are the last of the sequence's positions: row i sees keys j <= i + k_lens[s] - q_lens[s], and a row
 * that sees none gets zeros and a log-sum-exp of -infinity. Lengths may be 0. Built once per batch and kept
 * for all layers and all calls of it, on any stream. Blocks (the plan's copy); not during stream capture.
 * Errors: RIS_ERR_INVALID (n_seqs outside [1, 65535], a negative length, more than 2^31 - 65537 tokens),
 * RIS_ERR_OOM, RIS_ERR_CUDA. On error *out is NULL.
 * ris_pack_info: any output may be NULL. ris_pack_free: gives the plan back on the stream it was built on,
 * behind every call with the pack that was queued before, on whatever stream. Calls captured into a graph
 * are not among them: a graph must not be replayed once a pack in it was freed, nor the pack freed before
 * the last replay has finished. */
typedef struct ris_pack_s *ris_pack_t;
ris_status ris_pack_create(const int64_t *q_lens, const int64_t *k_lens, int32_t n_seqs, ris_pack_t *out, void *stream);
ris_status ris_pack_info(ris_pack_t pack, int32_t *n_seqs, int64_t *q_total, int64_t *k_total, int64_t *q_longest,
                         int64_t *k_longest);
ris_status ris_pack_free(ris_pack_t pack);

/* Rotate q [n][heads][head_dim] and k [n][kv_heads][head_dim] (k may be NULL with kv_heads 0) at given
 * positions, rotate-half pairs (c, c + D/2), then scale by the rope's mscale. Token i's heads start at
 * q + i * q_stride (elements, a multiple of 16 bytes, at least heads * head_dim: the rows of a fused
 * projection); q_out and k_out are contiguous, and may be q and k where those are contiguous.
 * positions: DEVICE int32 [axes][n], of either sign. sections: HOST [axes], 1 <= axes <= 4: how many of the
 * head_dim / 2 frequencies follow each axis (time, height, width), sections[0] first, or with
 * interleaved = 1 frequency c follows axis c mod axes while c / axes < sections[that axis], else axis 0. One
 * axis with sections[0] = head_dim / 2 is ordinary RoPE at any positions (packed prompts, a batch's next tokens). The
 * extension factor is resolved for n_ctx tokens. inverse = 1 turns backwards: the transposed
 * map, which takes the gradient of q_out and k_out to that of q and k. Angles as in
 * ris_attention_masked's own rotation; fp32 arithmetic, bf16 results rounded to nearest even.
 * Errors: RIS_ERR_INVALID (rope NULL or NONE, head_dim not 64 or 128, sections that do not sum to head_dim / 2). */
ris_status ris_rope_axes(const void *q, const void *k, void *q_out, void *k_out, int32_t dtype, int64_t n, int32_t heads,
                         int32_t kv_heads, int32_t head_dim, int64_t q_stride, int64_t k_stride, const int32_t *positions,
                         int32_t axes, const int32_t *sections, int32_t interleaved, int64_t n_ctx, const ris_rope_cfg *rope,
                         int32_t inverse, void *stream);

/* Causal attention over the sequences of a pack: q [q_total][heads][head_dim], k and v [k_total][kv_heads]
 * [head_dim] as given (rotated by the caller), token strides in elements as in ris_rope_axes;
 * out [q_total][heads][head_dim] contiguous; scores scaled by 1 / sqrt(head_dim).
 * lse: optional [heads][q_total] natural-log sum of exp of the scaled scores.
 * weight_rows W > 0 with key_weight [kv_heads][k_total]: the attention weight that each key got from the
 * last W rows of its sequence (all rows where there are fewer), summed over the query heads of its KV head: what
 * ris_cache4_append takes as the first of a slot's accumulated weight. W = 0: key_weight NULL; it may be
 * NULL where no sequence has a key.
 * head_dim in {64, 128}, any heads / kv_heads, fp32 or bf16. A key that a row does not see takes no part in
 * it, whatever it holds, and no prompt or KV head takes bits from another.
 * Precision: fp32 inputs never use a narrower product. bf16 inputs, whatever out_dtype is: exact products of
 * q and k summed in fp32; softmax statistics in fp32; a weight as fp16, with its 11 bits down to 2^-21 of the
 * row's largest; values as fp16 scaled by a power of two of their (sequence, KV head), exact down to 2^-30 of
 * its largest, and to 2^-12 of the key's own largest where that lies lower. Where the keys' largest values of
 * a (sequence, KV head) lie more than 2^26 apart or are not finite, and for rows of scores beyond 2^23, the
 * rows are computed on the FP32 pipe instead: about a hundred times slower.
 * Errors: RIS_ERR_INVALID, RIS_ERR_UNSUPPORTED (more row tiles x heads than a grid holds), RIS_ERR_OOM,
 * RIS_ERR_CUDA. */
ris_status ris_attention_packed(ris_pack_t pack, const void *q, const void *k, const void *v, void *out, int32_t heads,
                                int32_t kv_heads, int32_t head_dim, int64_t q_stride, int64_t k_stride, int64_t v_stride,
                                int32_t dtype, int32_t out_dtype, float *lse, int32_t weight_rows, float *key_weight,
                                void *stream);

/* A K/V cache held in 4 bits: caller-owned DEVICE arrays, each 16-byte aligned. Sequence b holds the
 * slots 0 .. length[b] - 1 of every KV head; the slots of a head need not be in the order of their
 * positions, and after an eviction differ from head to head.
 *   A row of head_dim values is cut into groups of 32. A group's scale is bf16(max |x| * fl32(1/6)) (NaN
 *   where a value is not finite: the group then stands for NaN); a value is stored as the e2m1 code (0, 0.5,
 *   1, 1.5, 2, 3, 4, 6, the value's sign in bit 3, also of -0) nearest to x / scale in fp32, ties to the even
 *   code, at most 6. Two codes make a byte, the even element in the low half. With i the byte's number in natural order, n = head_dim / 32 and m = head_dim / 16, it lies at
 *     keys    4 (((i / 4) mod 4) n + i / 16) + i mod 4,      values  (i mod 8) m + i / 8.
 * capacity is a multiple of 16; slots at and past length[b] may hold anything. `sync` is zeroed by the
 * caller once; every call leaves it zero. Calls on one cache must be ordered on the GPU. */
typedef struct {
    int32_t batch;     /* sequences, 1 .. 65535 */
    int32_t kv_heads;  /* 1 .. 4096 */
    int32_t head_dim;  /* 64 or 128 */
    int32_t reserved;  /* must be 0 */
    int64_t capacity;  /* slots of a sequence and head, a multiple of 16, at most 2^30 */
    uint8_t *k, *v;            /* [batch][kv_heads][capacity][head_dim / 2] codes */
    void *k_scale, *v_scale;   /* bf16 [batch][kv_heads][capacity][head_dim / 32] */
    int32_t *pos;              /* [batch][kv_heads][capacity] position of the slot's token */
    float *weight;             /* [batch][kv_heads][capacity] accumulated attention weight */
    int32_t *length;           /* [batch] slots in use */
    uint32_t *sync;            /* 4 words */
} ris_cache4;

/* Append the rows of a pack (its q side; sequence s to row s of the batch) to the cache: k and v
 * [q_total][kv_heads][head_dim], rotated, token strides in elements; positions: DEVICE int32 [q_total];
 * weight: optional DEVICE [kv_heads][q_total] (else 0). Token i of sequence b goes to slot start[b] + i and
 * length[b] becomes start[b] + q_lens[b], cut to 0 .. capacity; start NULL: after the slots in use. start (DEVICE int32 [batch]) must not be the cache's length.
 * Tokens past the capacity (or at a negative slot) are left out and reported by ris_device_status as
 * RIS_ERR_INVALID. A pack of ones is a decode step's append. Errors: RIS_ERR_INVALID, RIS_ERR_CUDA. */
ris_status ris_cache4_append(const ris_cache4 *cache, ris_pack_t pack, const void *k, const void *v, int64_t k_stride,
                             int64_t v_stride, int32_t dtype, const int32_t *positions, const float *weight,
                             const int32_t *start, void *stream);

/* The values that slots first[b] .. first[b] + count - 1 stand for (first NULL: 0; DEVICE int32 [batch]), exactly:
 * k and v fp32 [batch][kv_heads][count][head_dim]; zeros for slots that are not in use. */
ris_status ris_cache4_read(const ris_cache4 *cache, const int32_t *first, int64_t count, float *k, float *v, void *stream);

/* One token's attention per sequence over every slot in use: q [batch][heads][head_dim] (rotated), out the
 * same shape (out_dtype), lse optional [batch][heads]. A sequence without slots gets zeros and -infinity.
 * longest: an upper bound of the lengths that the caller knows (slots past it take no part), 0 for the
 * capacity: it sizes the grid and the scratch, so nothing in the launch depends on the lengths and a
 * captured graph can be replayed as they grow.
 * weight_out (optional, [batch][kv_heads][capacity]): weight_in + the weights of this token, summed over
 * the query heads of the KV head, for every slot in use (others untouched); weight_in NULL counts as 0 and
 * may be weight_out (the cache's own weight array, to add up in place).
 * Precision: the query as fp16 scaled by its head's largest element, in two parts for fp32 inputs (elements
 * below 2^-26 of the largest lose bits); scores, weights and sums in fp32. Weight times value scale goes
 * through one fp16 for bf16 outputs, two for fp32 outputs, with all bits down to 2^-18 of the largest that a
 * slot adds to the same query head and group of 32 channels. A group that stands for NaN makes those channels
 * NaN in its KV head's outputs; other groups, lse and weight_out do not depend on it.
 * Errors: RIS_ERR_INVALID, RIS_ERR_UNSUPPORTED (weights over more than 4096 query heads of a KV head, batch x
 * kv_heads past 2^24), RIS_ERR_OOM, RIS_ERR_CUDA. */
ris_status ris_cache4_attend(const ris_cache4 *cache, const void *q, int32_t heads, int32_t dtype, int32_t out_dtype,
                             int64_t longest, void *out, float *lse, const float *weight_in, float *weight_out, void *stream);

/* Cut every (sequence, KV head) of src with more than `budget` slots back to `budget`, into dst (another cache
 * of the same batch, kv_heads and head_dim with capacity >= budget, or src itself). Kept are the first `budget`
 * slots in this order: those with a position above the newest of the head - `recent`, then by weight
 * (NaN last), then by slot. A kept slot below the budget keeps its place; the i-th kept one at or above it
 * takes the i-th freed place below it. kept: DEVICE int32 [batch][kv_heads][budget], the source slot of each
 * place, -1 where there is none. dst's lengths become min(length, budget); its slots past that are untouched.
 * 0 <= recent < budget. Errors: RIS_ERR_INVALID, RIS_ERR_OOM, RIS_ERR_CUDA. */
ris_status ris_cache4_evict(const ris_cache4 *src, const ris_cache4 *dst, int32_t budget, int32_t recent, int32_t *kept,
                            void *stream);

/* ---- Normed heads, and a cache in pages ---------------------------------------------------------
 * The serving path of models that norm their queries and keys, and of servers that hand out memory by the
 * page (the paper has no counterpart).
 *
 * RMS norm of every head of q [n][heads][head_dim] and k [n][kv_heads][head_dim] (k may be NULL with kv_heads
 * 0), then the rotation to the token's position, in one pass: with r = (mean of the head's x^2 + eps)^-1/2,
 * z = x r weight; of z's first rot_dim channels (a multiple of 16; 0: head_dim) the pairs (c, c + rot_dim / 2),
 * or with pairs = 1 the neighbours (2c, 2c + 1), are turned by the angle of frequency c at positions[i] and
 * scaled by the rope's mscale; the other channels are z. The frequencies are those of a head of rot_dim
 * channels, their extension factor resolved for n_ctx tokens (ris_rope_freqs). q_weight, k_weight: DEVICE
 * [head_dim] of `dtype`, NULL: that tensor is not normed. rope NULL or of kind NONE: no rotation (positions may
 * be NULL, rot_dim is 0). positions: DEVICE int32 [n], of either sign. All strides are elements from token to
 * token, as in ris_rope_axes; an output may be its input (with the same stride), so that rows of a fused
 * projection are normed in place, and else must not overlap it.
 * Statistics and products in fp32, angles good to 2^-51 of themselves and 2^-30 radians at any position (64-bit fractions of a turn); bf16
 * results rounded once, to nearest even.
 *
 * The gradient: dq, dk of q_out, k_out; gq, gk of q, k (gq may be dq or q, with the same stride, gk alike); gq_weight,
 * gk_weight fp32 [head_dim], for each weight that there is, summed over all tokens and heads in a fixed order (zeros
 * for n = 0). q, k are the call's inputs as they were (not asked for where there is no weight).
 * Errors: RIS_ERR_INVALID, RIS_ERR_OOM (gradient), RIS_ERR_CUDA. */
ris_status ris_norm_rope(const void *q, const void *k, void *q_out, void *k_out, int32_t dtype, int64_t n, int32_t heads,
                         int32_t kv_heads, int32_t head_dim, int64_t q_stride, int64_t k_stride, int64_t q_out_stride,
                         int64_t k_out_stride, const int32_t *positions, const void *q_weight, const void *k_weight, float eps,
                         int32_t rot_dim, int32_t pairs, int64_t n_ctx, const ris_rope_cfg *rope, void *stream);
ris_status ris_norm_rope_backward(const void *dq, const void *dk, const void *q, const void *k, void *gq, void *gk, float *gq_weight,
                                  float *gk_weight, int32_t dtype, int64_t n, int32_t heads, int32_t kv_heads, int32_t head_dim,
                                  int64_t dq_stride, int64_t dk_stride, int64_t q_stride, int64_t k_stride, int64_t gq_stride,
                                  int64_t gk_stride, const int32_t *positions, const void *q_weight, const void *k_weight, float eps,
                                  int32_t rot_dim, int32_t pairs, int64_t n_ctx, const ris_rope_cfg *rope, void *stream);

/* A K/V cache in pages of page_size slots: caller-owned DEVICE arrays. Slot t of sequence b, which is the
 * sequence's token t, lies in page table[b][t / page_size], and its head g there at
 *     k (v) + page * page_stride + g * head_stride + (t mod page_size) * slot_stride    (elements)
 * so that [pages][kv_heads][page_size][head_dim], [pages][page_size][kv_heads][head_dim] and pools of keys
 * and values side by side all do. Sequences may share pages that none of them writes. Entries of the table
 * that a call does not reach may hold anything, and so may slots at and past length[b]. Calls on one cache
 * must be ordered on the GPU. */
typedef struct {
    int32_t batch;      /* sequences, 1 .. 65535 */
    int32_t kv_heads;   /* 1 .. 4096 */
    int32_t head_dim;   /* 64 or 128 */
    int32_t page_size;  /* a power of two, 16 .. 1024 */
    int32_t dtype;      /* RIS_F32 or RIS_BF16 */
    int32_t n_pages;    /* of the pools */
    int32_t table_len;  /* pages that a sequence can have; table_len * page_size <= 2^30 */
    int32_t reserved;   /* must be 0 */
    int64_t page_stride, head_stride, slot_stride;  /* each at least head_dim and a multiple of 16 bytes */
    void *k, *v;        /* 16-byte aligned */
    const int32_t *table;  /* [batch][table_len] */
    int32_t *length;    /* [batch] slots in use */
} ris_paged;

/* Append the rows of a pack (its q side; sequence s to row s of the batch): k and v [q_total][kv_heads]
 * [head_dim] of the cache's dtype, token strides in elements. Token i of sequence b goes to slot start[b] + i and length[b]
 * becomes start[b] + q_lens[b], cut to 0 .. the sequence's slots; start NULL: after the slots in use. start (DEVICE
 * int32 [batch]) must not be the cache's length. Tokens at a negative slot, past the table or in an entry that is
 * no page are left out and reported by ris_device_status as RIS_ERR_INVALID. A pack of ones is a decode step's append.
 * Errors: RIS_ERR_INVALID, RIS_ERR_CUDA. */
ris_status ris_paged_append(const ris_paged *cache, ris_pack_t pack, const void *k, const void *v, int64_t k_stride, int64_t v_stride,
                            const int32_t *start, void *stream);

/* Attention of a pack's rows (its q side) over the pages: q [q_total][heads][head_dim] (rotated), token stride
 * in elements; out [q_total][heads][head_dim] contiguous and apart from q, both of the cache's dtype; lse optional
 * [heads][q_total]; scores scaled by 1 / sqrt(head_dim). The rows are the last of their sequence's slots in use
 * (append them first): row i of sequence b is at p = length[b] - q_lens[b] + i and sees the keys j <= p that
 * have j > p - window or j < anchors; window 0: all of them (anchors is 0). Pages that no row sees are not
 * read, nor are their table entries. A row that sees no key (p < 0) gets zeros and a log-sum-exp of -infinity.
 * longest: an upper bound of the lengths that the caller knows (longer ones count as that long), 0 for the
 * table's. Nothing in the launches depends on the lengths, so a captured graph can be replayed as they grow.
 * One token, a few drafted ones and chunks of prompts may stand in one pack, any heads / kv_heads.
 * An entry of the table that is needed and no page is reported by ris_device_status as RIS_ERR_INVALID (the rows
 * that see it are then undefined). A key that a row does not see takes no part in it, whatever it holds.
 * fp32: products and sums in fp32. bf16: exact products, fp32 sums, each weight rounded once. Where a row sees a value that is not finite, or another
 * row of its tile does, or its largest weight is more than 2^100 times that of the first keys it is given (of its window, or of a share of its keys:
 * that can be one), a thread block does its share of the call twice; rows of scores past 2^28 are computed in fp32, slowly. Rows without such a value
 * or score come out the same, whatever stands beside them in the call.
 * Errors: RIS_ERR_INVALID, RIS_ERR_OOM, RIS_ERR_CUDA. */
ris_status ris_paged_attend(const ris_paged *cache, ris_pack_t pack, const void *q, int64_t q_stride, int32_t heads, int32_t window,
                            int32_t anchors, int64_t longest, void *out, float *lse, void *stream);

/* ---- Measurement support (the paper has no counterpart) -------------------------------------
 * Small kernels that measure the ceilings the attention kernels are compared against, for the
 * current device. Each allocates its own device buffers, runs on `stream` (NULL: legacy default
 * stream), synchronises it and frees what it allocated; none belongs on a hot path.
 *
 * ris_probe_l2_read: read bandwidth in GB/s (1e9 B/s) over a device buffer of `working_set`
 * bytes (1 MiB .. 4 GiB, rounded down to 256 B) that is read repeatedly, best of five launches
 * after one untimed launch. pattern 0: every thread streams 16-byte loads with a grid-wide
 * stride; pattern 1: groups of 16 threads read whole 256-byte rows at pseudo-random row
 * indices (the access pattern of the row-gathering attention kernels). Both load with .cg
 * (cached in L2 only), so a working set below the L2 size measures L2 and one well above it
 * measures HBM. Errors: RIS_ERR_INVALID (NULL gbs, size or pattern out of range), RIS_ERR_CUDA.
 *
 * ris_probe_ffma: FP32 fused multiply-add throughput in TFLOP/s (2 FLOPs per FFMA), eight
 * independent chains per thread, four 512-thread blocks per SM. Errors: RIS_ERR_INVALID,
 * RIS_ERR_CUDA.
 *
 * ris_probe_l2_bytes: L2 size in bytes as the driver reports it (cudaDevAttrL2CacheSize).
 *
 * ris_memory_stats: bytes in use now and the high-water mark of the current device's default
 * stream-ordered memory pool, from which this library takes its masks and per-call scratch
 * (the allocation-free entry point's fixed scratch is not counted). Other users of that pool
 * in the same process are counted too. reset_high_water != 0 resets the mark to zero after
 * reading it. Errors: RIS_ERR_INVALID (NULL outputs), RIS_ERR_CUDA. */
ris_status ris_probe_l2_read(int64_t working_set, int32_t pattern, double *gbs, void *stream);
ris_status ris_probe_ffma(double *tflops, void *stream);
ris_status ris_probe_l2_bytes(int64_t *bytes);
ris_status ris_memory_stats(int64_t *in_use, int64_t *high_water, int32_t reset_high_water);

/* Text of the calling thread's last error ("" if none). The string is owned by the library. */
const char *ris_last_error(void);

/* Number of kernels this library has launched since it was loaded (all threads). */
int64_t ris_launch_count(void);

/* Library version string. */
const char *ris_version(void);

#ifdef __cplusplus
}
#endif

#endif /* RIS_H */
