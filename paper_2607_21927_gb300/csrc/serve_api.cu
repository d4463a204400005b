// C ABI of the serving operators: packed prompts, positions on several axes, the 4-bit cache, normed and
// turned heads, and the cache in pages. Argument checks, the plan of a pack, scratch and the launches; the
// work is in rope_axes.cu, norm_rope.cu, attn_packed.cu, attn_packed_f32.cu, cache4.cu, cache4_evict.cu, paged.cu
// and attn_paged.cu.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <mutex>
#include <new>
#include <utility>
#include <vector>

#include "serve.h"

using namespace ris;

struct ris_pack_s {
    int32_t n_seqs = 0;
    int64_t q_total = 0, k_total = 0, q_longest = 0, k_longest = 0;
    void *mem = nullptr;  // device: everything below
    int32_t *q_off = nullptr, *seq_of = nullptr;
    PackItem *items = nullptr, *pairs = nullptr, *key_items = nullptr;  // of 128 rows, 256 rows, 128 keys
    PackRun *runs = nullptr;
    int32_t n_items = 0, n_pairs = 0, n_key_items = 0, n_runs = 0;
    int64_t key_tiles = 0;  // of 128 x 128 that the items of 128 rows see
    cudaStream_t stream = nullptr;
    // Streams other than its own that calls with it were queued on, each with an event behind the last of
    // them: its memory is given back behind these.
    std::mutex mu;
    std::vector<std::pair<cudaStream_t, cudaEvent_t>> used;
    bool unknown = false;  // a use could not be noted: the device is waited for
};

namespace {

// Errors go to the same per-thread text that ris_last_error() returns.
ris_status fail(ris_status st, const char *fmt, ...)
{
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof(buf), fmt, ap);
    va_end(ap);
    set_error_text(buf);
    return st;
}

ris_status cuda_fail(cudaError_t e, const char *what)
{
    cudaGetLastError();  // clear a sticky launch error of this thread
    return fail(e == cudaErrorMemoryAllocation ? RIS_ERR_OOM : RIS_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

#define RIS_CUDA(call)                                      \
    do {                                                    \
        cudaError_t e_ = (call);                            \
        if (e_ != cudaSuccess) return cuda_fail(e_, #call); \
    } while (0)

#define RIS_TRY(expr)                  \
    do {                               \
        ris_status st_ = (expr);       \
        if (st_ != RIS_OK) return st_; \
    } while (0)

struct Scratch {
    void *p = nullptr;
    cudaStream_t s = nullptr;
    cudaError_t alloc(size_t bytes, cudaStream_t st)
    {
        s = st;
        return library_alloc(&p, bytes, st);
    }
    ~Scratch()
    {
        if (p) cudaFreeAsync(p, s);
    }
};

// Notes that a call queues work with the pack on `s`, behind that work: when the call returns, whether it
// succeeds or not.
struct PackUse {
    ris_pack_s *pack;
    cudaStream_t s;
    ~PackUse()
    {
        // (the per-thread default stream is another one in each thread: one handle says too little)
        const bool one = s != cudaStreamPerThread;
        if (s == pack->stream && one) return;
        cudaStreamCaptureStatus st = cudaStreamCaptureStatusNone;
        cudaError_t e = cudaStreamIsCapturing(s, &st);
        if (e == cudaSuccess && st != cudaStreamCaptureStatusNone) return;  // (a graph's uses are the caller's to order)
        std::lock_guard<std::mutex> lk(pack->mu);
        cudaEvent_t ev = nullptr;
        for (const auto &u : pack->used)
            if (u.first == s) ev = u.second;
        if (e == cudaSuccess && one && ev == nullptr) {
            e = cudaEventCreateWithFlags(&ev, cudaEventDisableTiming);
            if (e == cudaSuccess) try {
                    pack->used.emplace_back(s, ev);
                } catch (...) {  // host memory
                    cudaEventDestroy(ev);
                    e = cudaErrorMemoryAllocation;
                }
        }
        if (e == cudaSuccess && one) e = cudaEventRecord(ev, s);
        if (e != cudaSuccess || !one) {
            cudaGetLastError();
            pack->unknown = true;
        }
    }
};

constexpr size_t room(size_t bytes) { return (bytes + 255) & ~size_t(255); }

bool aligned(const void *p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

ris_status check_ptr(const void *p, const char *what)
{
    if (p == nullptr) return fail(RIS_ERR_INVALID, "%s is NULL", what);
    if (!aligned(p, 16)) return fail(RIS_ERR_INVALID, "%s is not 16-byte aligned", what);
    return RIS_OK;
}

ris_status check_dtype(int32_t dt, const char *what)
{
    if (dt != RIS_F32 && dt != RIS_BF16) return fail(RIS_ERR_INVALID, "%s %d is neither F32 nor BF16", what, dt);
    return RIS_OK;
}

ris_status check_heads(int32_t heads, int32_t kv_heads, int32_t head_dim)
{
    if (heads < 1 || kv_heads < 1 || heads > 65535) return fail(RIS_ERR_INVALID, "heads and kv_heads must be in [1, 65535]");
    if (heads % kv_heads != 0) return fail(RIS_ERR_INVALID, "heads %d not a multiple of kv_heads %d", heads, kv_heads);
    if (head_dim != 64 && head_dim != 128) return fail(RIS_ERR_INVALID, "head_dim %d not in {64, 128}", head_dim);
    return RIS_OK;
}

// Elements from one token's heads to the next's: whole heads apart, in steps of 16 bytes.
ris_status check_stride(int64_t stride, int64_t row, int32_t dtype, const char *what)
{
    const int64_t unit = dtype == RIS_F32 ? 4 : 8;
    if (stride < row || stride > (int64_t(1) << 31) || stride % unit != 0)
        return fail(RIS_ERR_INVALID, "%s %lld must be at least %lld, at most 2^31 and a multiple of 16 bytes", what,
                    (long long)stride, (long long)row);
    return RIS_OK;
}

ris_status check_cache(const ris_cache4 *c, const char *what)
{
    if (c == nullptr) return fail(RIS_ERR_INVALID, "%s is NULL", what);
    if (c->batch < 1 || c->batch > kMaxPackSeqs) return fail(RIS_ERR_INVALID, "%s: batch %d outside [1, %d]", what, c->batch, kMaxPackSeqs);
    if (c->kv_heads < 1 || c->kv_heads > 4096) return fail(RIS_ERR_INVALID, "%s: kv_heads %d outside [1, 4096]", what, c->kv_heads);
    if (c->head_dim != 64 && c->head_dim != 128) return fail(RIS_ERR_INVALID, "%s: head_dim %d not in {64, 128}", what, c->head_dim);
    if (c->reserved != 0) return fail(RIS_ERR_INVALID, "%s: reserved must be 0", what);
    if (c->capacity < 16 || c->capacity % 16 != 0 || c->capacity > (int64_t(1) << 30))
        return fail(RIS_ERR_INVALID, "%s: capacity %lld must be a multiple of 16 in [16, 2^30]", what, (long long)c->capacity);
    const void *const p[] = {c->k, c->v, c->k_scale, c->v_scale, c->pos, c->weight, c->length, c->sync};
    const char *const name[] = {"k", "v", "k_scale", "v_scale", "pos", "weight", "length", "sync"};
    for (int i = 0; i < 8; ++i)
        if (p[i] == nullptr || !aligned(p[i], 16)) return fail(RIS_ERR_INVALID, "%s: %s is NULL or not 16-byte aligned", what, name[i]);
    return RIS_OK;
}

Cache4Args cache_args(const ris_cache4 *c)
{
    Cache4Args a{};
    a.k = c->k;
    a.v = c->v;
    a.k_scale = static_cast<uint16_t *>(c->k_scale);
    a.v_scale = static_cast<uint16_t *>(c->v_scale);
    a.pos = c->pos;
    a.weight = c->weight;
    a.length = c->length;
    a.B = c->batch;
    a.Hkv = c->kv_heads;
    a.D = c->head_dim;
    a.cap = c->capacity;
    return a;
}

double log2e_over_sqrt(int32_t head_dim) { return 1.4426950408889634074 / std::sqrt((double)head_dim); }

// Keys that the last of an item's `step` rows sees.
int64_t keys_of(const PackItem &it, int step)
{
    const int64_t last = std::min<int64_t>((int64_t)it.row + step, it.q_len) + it.k_len - it.q_len;
    return std::max<int64_t>(0, std::min<int64_t>(last, it.k_len));
}

// Head dim 128, bf16: whether a pack's row tiles see so many key tiles (24 on average, about 6,000 tokens
// of one prompt) that two CTAs sharing every key tile beat two independent ones on each SM, which finish a
// row tile and start the next one with less delay. us a call of 16,384 to 18,432 tokens, clusters / rows:
// prompts of 256 tokens 86 / 41, of 1024 107 / 67, of 4096 183 / 163, of 6144 254 / 259, of 8192 275 / 299,
// of 16384 465 / 565 (12 / 2 heads; 8 / 8 heads: of 4096 138 / 126, of 8192 201 / 220).
bool packed_by_clusters(const ris_pack_s *pack) { return pack->key_tiles >= 24LL * pack->n_items; }

// The items of `step` rows (or keys) of every sequence; of rows, those with the most keys first, so that the
// short ones fill the tail of the grid.
std::vector<PackItem> items_of(const std::vector<int32_t> &q_off, const std::vector<int32_t> &k_off, bool keys, int step)
{
    std::vector<PackItem> v;
    for (size_t s = 0; s + 1 < q_off.size(); ++s) {
        PackItem it{};
        it.seq = (int32_t)s;
        it.q_base = q_off[s];
        it.q_len = q_off[s + 1] - q_off[s];
        it.k_base = k_off[s];
        it.k_len = k_off[s + 1] - k_off[s];
        const int32_t n = keys ? it.k_len : it.q_len;
        for (int64_t r = 0; r < n; r += step) {
            it.row = (int32_t)r;
            v.push_back(it);
        }
    }
    if (!keys)
        std::stable_sort(v.begin(), v.end(), [step](const PackItem &x, const PackItem &y) { return keys_of(x, step) > keys_of(y, step); });
    return v;
}

// Runs of the keys: whole key items, so long that there are about kPackRuns of them.
std::vector<PackRun> runs_of(const std::vector<int32_t> &k_off)
{
    const int64_t total = k_off.back(), step = std::max<int64_t>(1, (total + (int64_t)kPackRuns * kPackKeys - 1) / ((int64_t)kPackRuns * kPackKeys)) * kPackKeys;
    std::vector<PackRun> v;
    for (size_t s = 0; s + 1 < k_off.size(); ++s) {
        PackRun r{};
        r.seq = (int32_t)s;
        r.run0 = (int32_t)v.size();
        r.run1 = (int32_t)(r.run0 + (k_off[s + 1] - k_off[s] + step - 1) / step);
        for (int64_t k = k_off[s]; k < k_off[s + 1]; k += step) {
            r.first = (int32_t)k;
            r.n = (int32_t)std::min<int64_t>(step, k_off[s + 1] - k);
            v.push_back(r);
        }
    }
    return v;
}

// What both directions of ris_norm_rope share: checks, and the arguments but for the tensors.
ris_status norm_rope_args(NormRopeArgs &a, int32_t dtype, int64_t n, int32_t heads, int32_t kv_heads, int32_t head_dim, const int32_t *positions,
                          const void *q_weight, const void *k_weight, float eps, int32_t rot_dim, int32_t pairs, int64_t n_ctx,
                          const ris_rope_cfg *rope)
{
    RIS_TRY(check_dtype(dtype, "dtype"));
    if (n < 0 || n > 2147483647LL) return fail(RIS_ERR_INVALID, "n=%lld outside [0, 2^31-1]", (long long)n);
    if (heads < 1 || kv_heads < 0 || heads > 65535 || kv_heads > 65535)
        return fail(RIS_ERR_INVALID, "heads must be in [1, 65535], kv_heads in [0, 65535]");
    if (head_dim != 64 && head_dim != 128) return fail(RIS_ERR_INVALID, "head_dim %d not in {64, 128}", head_dim);
    if (pairs != 0 && pairs != 1) return fail(RIS_ERR_INVALID, "pairs must be 0 or 1");
    if (!(eps >= 0.f) || !std::isfinite(eps)) return fail(RIS_ERR_INVALID, "eps must be finite and >= 0");
    if (kv_heads == 0 && k_weight != nullptr) return fail(RIS_ERR_INVALID, "k_weight without k");
    for (const void *w : {q_weight, k_weight})
        if (w != nullptr && !aligned(w, 16)) return fail(RIS_ERR_INVALID, "a weight is not 16-byte aligned");
    const bool turns = rope != nullptr && rope->kind != RIS_ROPE_NONE;
    if (!turns) {
        if (q_weight == nullptr && k_weight == nullptr) return fail(RIS_ERR_INVALID, "neither a weight nor a rotation");
        if (rot_dim != 0) return fail(RIS_ERR_INVALID, "rot_dim %d without a rotation", rot_dim);
    } else {
        if (rot_dim == 0) rot_dim = head_dim;
        if (rot_dim < 16 || rot_dim > head_dim || rot_dim % 16 != 0)
            return fail(RIS_ERR_INVALID, "rot_dim %d must be a multiple of 16 in [16, head_dim]", rot_dim);
        double f[kMaxHeadDimHalf], ms = 1.0;
        RIS_TRY(ris_rope_freqs(rope, n_ctx, rot_dim, f, &ms));
        if (n > 0 && (positions == nullptr || !aligned(positions, 4))) return fail(RIS_ERR_INVALID, "positions is NULL or misaligned");
        for (int c = 0; c < rot_dim / 2; ++c)  // as fractions of a turn in 2^-64
            a.turn[c] = (uint64_t)(f[c] * (18446744073709551616.0 / 6.283185307179586476925286766559));
        a.mscale = (float)ms;
    }
    a.heads[0] = heads, a.heads[1] = kv_heads;
    a.n = n;
    a.pos = positions;
    a.weight[0] = q_weight, a.weight[1] = k_weight;
    a.eps = eps;
    a.rot = rot_dim;
    return RIS_OK;
}

ris_status check_paged(const ris_paged *c)
{
    if (c == nullptr) return fail(RIS_ERR_INVALID, "cache is NULL");
    if (c->batch < 1 || c->batch > kMaxPackSeqs) return fail(RIS_ERR_INVALID, "batch %d outside [1, %d]", c->batch, kMaxPackSeqs);
    if (c->kv_heads < 1 || c->kv_heads > 4096) return fail(RIS_ERR_INVALID, "kv_heads %d outside [1, 4096]", c->kv_heads);
    if (c->head_dim != 64 && c->head_dim != 128) return fail(RIS_ERR_INVALID, "head_dim %d not in {64, 128}", c->head_dim);
    if (c->page_size < 16 || c->page_size > 1024 || (c->page_size & (c->page_size - 1)) != 0)
        return fail(RIS_ERR_INVALID, "page_size %d must be a power of two in [16, 1024]", c->page_size);
    RIS_TRY(check_dtype(c->dtype, "dtype"));
    if (c->n_pages < 1 || c->table_len < 1 || c->reserved != 0) return fail(RIS_ERR_INVALID, "n_pages and table_len must be positive, reserved 0");
    if ((int64_t)c->table_len * c->page_size > (int64_t(1) << 30))
        return fail(RIS_ERR_INVALID, "table_len x page_size = %lld slots, at most 2^30", (long long)c->table_len * c->page_size);
    const int64_t unit = c->dtype == RIS_F32 ? 4 : 8;
    for (int64_t x : {c->page_stride, c->head_stride, c->slot_stride})
        if (x < c->head_dim || x % unit != 0 || x > (int64_t(1) << 36))
            return fail(RIS_ERR_INVALID, "a stride of %lld must be at least head_dim, a multiple of 16 bytes and at most 2^36", (long long)x);
    RIS_TRY(check_ptr(c->k, "k"));
    RIS_TRY(check_ptr(c->v, "v"));
    if (c->table == nullptr || !aligned(c->table, 4)) return fail(RIS_ERR_INVALID, "table is NULL or misaligned");
    if (c->length == nullptr || !aligned(c->length, 4)) return fail(RIS_ERR_INVALID, "length is NULL or misaligned");
    return RIS_OK;
}

PagedArgs paged_args(const ris_paged *c)
{
    PagedArgs a{};
    a.k = c->k, a.v = c->v;
    a.page_stride = c->page_stride, a.head_stride = c->head_stride, a.slot_stride = c->slot_stride;
    a.table = c->table;
    a.length = c->length;
    a.B = c->batch, a.Hkv = c->kv_heads, a.D = c->head_dim;
    while ((1 << a.page_log2) < c->page_size) ++a.page_log2;
    a.n_pages = c->n_pages, a.table_len = c->table_len;
    return a;
}

}  // namespace

extern "C" {

// ---------------------------------------------------------------- packs
ris_status ris_pack_create(const int64_t *q_lens, const int64_t *k_lens, int32_t n_seqs, ris_pack_t *out, void *stream)
{
    if (out == nullptr) return fail(RIS_ERR_INVALID, "out is NULL");
    *out = nullptr;
    if (q_lens == nullptr) return fail(RIS_ERR_INVALID, "q_lens is NULL");
    if (n_seqs < 1 || n_seqs > kMaxPackSeqs) return fail(RIS_ERR_INVALID, "n_seqs %d outside [1, %d]", n_seqs, kMaxPackSeqs);
    constexpr int64_t kMost = 2147483647LL - 65536;  // tokens of a pack: every row index, rounded up, is an int
    int64_t nq = 0, nk = 0;
    for (int32_t s = 0; s < n_seqs; ++s) {
        const int64_t a = q_lens[s], b = k_lens != nullptr ? k_lens[s] : a;
        if (a < 0 || b < 0 || a > kMost || b > kMost) return fail(RIS_ERR_INVALID, "lengths of sequence %d: %lld, %lld", s, (long long)a, (long long)b);
        nq += a;
        nk += b;
        if (nq > kMost || nk > kMost) return fail(RIS_ERR_INVALID, "more than 2^31 - 65537 tokens");
    }
    ris_pack_s *p = nullptr;
    try {
        std::vector<int32_t> q_off(n_seqs + 1), k_off(n_seqs + 1), seq_of((size_t)nq);
        p = new ris_pack_s;
        p->n_seqs = n_seqs;
        for (int32_t s = 0; s < n_seqs; ++s) {
            const int64_t a = q_lens[s], b = k_lens != nullptr ? k_lens[s] : a;
            q_off[s + 1] = q_off[s] + (int32_t)a;
            k_off[s + 1] = k_off[s] + (int32_t)b;
            std::fill(seq_of.begin() + q_off[s], seq_of.begin() + q_off[s + 1], s);
            p->q_longest = std::max(p->q_longest, a);
            p->k_longest = std::max(p->k_longest, b);
        }
        p->q_total = nq;
        p->k_total = nk;
        const std::vector<PackItem> items = items_of(q_off, k_off, false, kPackRows), pairs = items_of(q_off, k_off, false, 2 * kPackRows),
                                    keys = items_of(q_off, k_off, true, kPackKeys);
        for (const PackItem &it : items) p->key_tiles += (keys_of(it, kPackRows) + kPackKeys - 1) / kPackKeys;
        p->n_items = (int32_t)items.size();
        p->n_pairs = (int32_t)pairs.size();
        p->n_key_items = (int32_t)keys.size();
        const std::vector<PackRun> runs = runs_of(k_off);
        p->n_runs = (int32_t)runs.size();
        cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
        p->stream = s;
        const size_t off_b = room(sizeof(int32_t) * q_off.size()), seq_b = room(sizeof(int32_t) * seq_of.size()),
                     item_b = room(sizeof(PackItem) * items.size()), pair_b = room(sizeof(PackItem) * pairs.size()),
                     key_b = room(sizeof(PackItem) * keys.size()), run_b = room(sizeof(PackRun) * runs.size());
        cudaError_t e = library_alloc(&p->mem, off_b + seq_b + item_b + pair_b + key_b + run_b, s);
        char *d = static_cast<char *>(p->mem);
        auto put = [&](const void *src, size_t bytes) {
            if (e == cudaSuccess && bytes > 0) e = cudaMemcpyAsync(d, src, bytes, cudaMemcpyHostToDevice, s);
        };
        p->q_off = reinterpret_cast<int32_t *>(d);
        put(q_off.data(), sizeof(int32_t) * q_off.size());
        d += off_b;
        p->seq_of = reinterpret_cast<int32_t *>(d);
        put(seq_of.data(), sizeof(int32_t) * seq_of.size());
        d += seq_b;
        p->items = reinterpret_cast<PackItem *>(d);
        put(items.data(), sizeof(PackItem) * items.size());
        d += item_b;
        p->pairs = reinterpret_cast<PackItem *>(d);
        put(pairs.data(), sizeof(PackItem) * pairs.size());
        d += pair_b;
        p->key_items = reinterpret_cast<PackItem *>(d);
        put(keys.data(), sizeof(PackItem) * keys.size());
        d += key_b;
        p->runs = reinterpret_cast<PackRun *>(d);
        put(runs.data(), sizeof(PackRun) * runs.size());
        // the host arrays end with this call: the copies out of them must have been taken
        if (e == cudaSuccess) e = cudaStreamSynchronize(s);
        if (e != cudaSuccess) {
            if (p->mem) cudaFreeAsync(p->mem, s);
            delete p;
            return cuda_fail(e, "the plan of a pack");
        }
    } catch (...) {  // host memory
        delete p;
        return fail(RIS_ERR_OOM, "no host memory for the plan of a pack");
    }
    *out = p;
    return RIS_OK;
}

ris_status ris_pack_info(ris_pack_t pack, int32_t *n_seqs, int64_t *q_total, int64_t *k_total, int64_t *q_longest,
                         int64_t *k_longest)
{
    if (pack == nullptr) return fail(RIS_ERR_INVALID, "pack is NULL");
    if (n_seqs) *n_seqs = pack->n_seqs;
    if (q_total) *q_total = pack->q_total;
    if (k_total) *k_total = pack->k_total;
    if (q_longest) *q_longest = pack->q_longest;
    if (k_longest) *k_longest = pack->k_longest;
    return RIS_OK;
}

ris_status ris_pack_free(ris_pack_t pack)
{
    if (pack == nullptr) return RIS_OK;
    cudaError_t e = cudaSuccess;
    for (const auto &u : pack->used)
        if (e == cudaSuccess) e = cudaStreamWaitEvent(pack->stream, u.second, 0);
    if (pack->unknown || e != cudaSuccess) {
        cudaGetLastError();
        e = cudaDeviceSynchronize();
    }
    if (pack->mem) {
        const cudaError_t e2 = cudaFreeAsync(pack->mem, pack->stream);
        if (e == cudaSuccess) e = e2;
    }
    for (const auto &u : pack->used) cudaEventDestroy(u.second);
    delete pack;
    if (e != cudaSuccess) return cuda_fail(e, "cudaFreeAsync");
    return RIS_OK;
}

// ---------------------------------------------------------------- positions
ris_status ris_rope_axes(const void *q, const void *k, void *q_out, void *k_out, int32_t dtype, int64_t n, int32_t heads,
                         int32_t kv_heads, int32_t head_dim, int64_t q_stride, int64_t k_stride, const int32_t *positions,
                         int32_t axes, const int32_t *sections, int32_t interleaved, int64_t n_ctx, const ris_rope_cfg *rope,
                         int32_t inverse, void *stream)
{
    RIS_TRY(check_dtype(dtype, "dtype"));
    if (n < 0 || n > 2147483647LL) return fail(RIS_ERR_INVALID, "n=%lld outside [0, 2^31-1]", (long long)n);
    if (heads < 1 || kv_heads < 0 || heads > 65535 || kv_heads > 65535)
        return fail(RIS_ERR_INVALID, "heads must be in [1, 65535], kv_heads in [0, 65535]");
    if (head_dim != 64 && head_dim != 128) return fail(RIS_ERR_INVALID, "head_dim %d not in {64, 128}", head_dim);
    if (axes < 1 || axes > kMaxAxes) return fail(RIS_ERR_INVALID, "axes %d outside [1, %d]", axes, kMaxAxes);
    if (sections == nullptr) return fail(RIS_ERR_INVALID, "sections is NULL");
    if ((interleaved != 0 && interleaved != 1) || (inverse != 0 && inverse != 1))
        return fail(RIS_ERR_INVALID, "interleaved and inverse must be 0 or 1");
    int64_t sum = 0;
    for (int32_t x = 0; x < axes; ++x) {
        if (sections[x] < 0) return fail(RIS_ERR_INVALID, "sections[%d] = %d", x, sections[x]);
        sum += sections[x];
    }
    if (sum != head_dim / 2)
        return fail(RIS_ERR_INVALID, "the sections hold %lld frequencies, not head_dim / 2 = %d", (long long)sum, head_dim / 2);
    if (rope == nullptr || rope->kind == RIS_ROPE_NONE) return fail(RIS_ERR_INVALID, "rope is NULL or of kind NONE");
    RopeAxesArgs a{};
    double f[kMaxHeadDimHalf], ms = 1.0;
    RIS_TRY(ris_rope_freqs(rope, n_ctx, head_dim, f, &ms));
    if (n > 0) {
        RIS_TRY(check_ptr(q, "q"));
        RIS_TRY(check_ptr(q_out, "q_out"));
        if (kv_heads > 0) {
            RIS_TRY(check_ptr(k, "k"));
            RIS_TRY(check_ptr(k_out, "k_out"));
        }
        if (positions == nullptr || !aligned(positions, 4)) return fail(RIS_ERR_INVALID, "positions is NULL or misaligned");
        RIS_TRY(check_stride(q_stride, (int64_t)heads * head_dim, dtype, "q_stride"));
        if (kv_heads > 0) RIS_TRY(check_stride(k_stride, (int64_t)kv_heads * head_dim, dtype, "k_stride"));
        if ((q == q_out && q_stride != (int64_t)heads * head_dim) ||
            (kv_heads > 0 && k == k_out && k_stride != (int64_t)kv_heads * head_dim))
            return fail(RIS_ERR_INVALID, "in place only where the heads of a token follow the last one's");
    }
    if (n == 0) return RIS_OK;
    for (int c = 0; c < head_dim / 2; ++c)  // as fractions of a turn in 2^-64
        a.turn[c] = (uint64_t)(f[c] * (18446744073709551616.0 / 6.283185307179586476925286766559));
    if (interleaved) {
        // frequency c goes to axis c mod axes while that axis has any left, else to the first axis
        for (int c = 0; c < head_dim / 2; ++c) {
            const int x = c % axes;
            a.axis[c] = (uint8_t)(x > 0 && c / axes < sections[x] ? x : 0);
        }
    } else {
        for (int32_t x = 0, c = 0; x < axes; ++x)
            for (int32_t i = 0; i < sections[x]; ++i) a.axis[c++] = (uint8_t)x;
    }
    a.x[0] = q, a.x[1] = k;
    a.y[0] = q_out, a.y[1] = k_out;
    a.stride[0] = q_stride, a.stride[1] = k_stride;
    a.heads[0] = heads, a.heads[1] = kv_heads;
    a.n = n;
    a.D = head_dim;
    a.pos = positions;
    a.mscale = (float)ms;
    a.inverse = inverse;
    RIS_CUDA(launch_rope_axes(a, dtype, reinterpret_cast<cudaStream_t>(stream)));
    return RIS_OK;
}

// ---------------------------------------------------------------- packed prompts
ris_status ris_attention_packed(ris_pack_t pack, const void *q, const void *k, const void *v, void *out, int32_t heads,
                                int32_t kv_heads, int32_t head_dim, int64_t q_stride, int64_t k_stride, int64_t v_stride,
                                int32_t dtype, int32_t out_dtype, float *lse, int32_t weight_rows, float *key_weight,
                                void *stream)
{
    if (pack == nullptr) return fail(RIS_ERR_INVALID, "pack is NULL");
    RIS_TRY(check_heads(heads, kv_heads, head_dim));
    RIS_TRY(check_dtype(dtype, "dtype"));
    RIS_TRY(check_dtype(out_dtype, "out_dtype"));
    if (weight_rows < 0) return fail(RIS_ERR_INVALID, "weight_rows %d must be >= 0", weight_rows);
    if (weight_rows == 0 && key_weight != nullptr) return fail(RIS_ERR_INVALID, "key_weight without weight_rows");
    if (weight_rows > 0 && key_weight == nullptr && pack->k_total > 0) return fail(RIS_ERR_INVALID, "weight_rows without key_weight");
    if ((lse != nullptr && !aligned(lse, 16)) || (key_weight != nullptr && !aligned(key_weight, 16)))
        return fail(RIS_ERR_INVALID, "lse or key_weight is not 16-byte aligned");
    if (pack->q_total > 0) {
        RIS_TRY(check_ptr(q, "q"));
        RIS_TRY(check_ptr(out, "out"));
        RIS_TRY(check_stride(q_stride, (int64_t)heads * head_dim, dtype, "q_stride"));
    }
    if (pack->k_total > 0) {
        RIS_TRY(check_ptr(k, "k"));
        RIS_TRY(check_ptr(v, "v"));
        RIS_TRY(check_stride(k_stride, (int64_t)kv_heads * head_dim, dtype, "k_stride"));
        RIS_TRY(check_stride(v_stride, (int64_t)kv_heads * head_dim, dtype, "v_stride"));
    }
    if ((int64_t)pack->n_items * 4 * heads > 2147483647LL)
        return fail(RIS_ERR_UNSUPPORTED, "%d row tiles x %d heads are more than a grid holds", pack->n_items, heads);
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    PackedArgs a{};
    a.q = q, a.k = k, a.v = v;
    a.q_stride = q_stride, a.k_stride = k_stride, a.v_stride = v_stride;
    a.out = out;
    a.lse = lse;
    a.q_total = pack->q_total;
    a.k_total = pack->k_total;
    a.items = pack->items;
    a.n_items = pack->n_items;
    a.key_items = pack->key_items;
    a.n_key_items = pack->n_key_items;
    a.runs = pack->runs;
    a.n_runs = pack->n_runs;
    a.n_seqs = pack->n_seqs;
    a.Hq = heads;
    a.Hkv = kv_heads;
    a.G = heads / kv_heads;
    a.scale_log2 = (float)log2e_over_sqrt(head_dim);
    a.weight_rows = weight_rows;
    a.key_weight = key_weight;
    const bool tiles = dtype == RIS_BF16;
    const bool clusters = tiles && head_dim == 128 && packed_by_clusters(pack);
    if (clusters && (a.G & 1) != 0) {
        a.items = pack->pairs;
        a.n_items = pack->n_pairs;
    }
    const size_t stat_b = weight_rows > 0 ? room(sizeof(float2) * (size_t)heads * pack->q_total) : 0;
    const size_t tile_b = tiles ? packed_scratch_bytes(a, head_dim) : 0;
    const PackUse use{pack, s};
    Scratch mem;
    if (stat_b + tile_b > 0) RIS_CUDA(mem.alloc(stat_b + tile_b, s));
    if (weight_rows > 0) a.row_stat = static_cast<float2 *>(mem.p);
    if (pack->n_items > 0)
        RIS_CUDA(tiles ? launch_packed_tiles(a, head_dim, out_dtype, clusters, static_cast<char *>(mem.p) + stat_b, s)
                       : launch_packed_f32(a, head_dim, out_dtype, s));
    if (weight_rows > 0 && pack->n_key_items > 0)
        RIS_CUDA(tiles ? launch_packed_weights_tc(a, head_dim, s) : launch_packed_weights_f32(a, head_dim, s));
    return RIS_OK;
}

// ---------------------------------------------------------------- the 4-bit cache
ris_status ris_cache4_append(const ris_cache4 *cache, ris_pack_t pack, const void *k, const void *v, int64_t k_stride,
                             int64_t v_stride, int32_t dtype, const int32_t *positions, const float *weight,
                             const int32_t *start, void *stream)
{
    RIS_TRY(check_cache(cache, "cache"));
    if (pack == nullptr) return fail(RIS_ERR_INVALID, "pack is NULL");
    if (pack->n_seqs != cache->batch)
        return fail(RIS_ERR_INVALID, "the pack has %d sequences, the cache %d", pack->n_seqs, cache->batch);
    RIS_TRY(check_dtype(dtype, "dtype"));
    if (start != nullptr && (!aligned(start, 4) || start == cache->length))
        return fail(RIS_ERR_INVALID, "start is misaligned or the cache's own lengths (pass NULL for those)");
    if (pack->q_total == 0) {
        if (start != nullptr) RIS_CUDA(launch_cache4_start(cache_args(cache), start, reinterpret_cast<cudaStream_t>(stream)));
        return RIS_OK;
    }
    RIS_TRY(check_ptr(k, "k"));
    RIS_TRY(check_ptr(v, "v"));
    RIS_TRY(check_stride(k_stride, (int64_t)cache->kv_heads * cache->head_dim, dtype, "k_stride"));
    RIS_TRY(check_stride(v_stride, (int64_t)cache->kv_heads * cache->head_dim, dtype, "v_stride"));
    if (positions == nullptr || !aligned(positions, 4)) return fail(RIS_ERR_INVALID, "positions is NULL or misaligned");
    if (weight != nullptr && !aligned(weight, 4)) return fail(RIS_ERR_INVALID, "weight is misaligned");
    if (pack->q_total * cache->kv_heads > 32LL * 2147483647LL) return fail(RIS_ERR_UNSUPPORTED, "more rows than a grid holds");
    Cache4AppendArgs a{};
    a.c = cache_args(cache);
    a.k = k, a.v = v;
    a.k_stride = k_stride, a.v_stride = v_stride;
    a.positions = positions;
    a.weight = weight;
    a.start = start;
    a.off = pack->q_off;
    a.seq_of = pack->seq_of;
    a.total = pack->q_total;
    a.ticket = cache->sync;
    const PackUse use{pack, reinterpret_cast<cudaStream_t>(stream)};
    RIS_CUDA(launch_cache4_append(a, dtype, reinterpret_cast<cudaStream_t>(stream)));
    return RIS_OK;
}

ris_status ris_cache4_read(const ris_cache4 *cache, const int32_t *first, int64_t count, float *k, float *v, void *stream)
{
    RIS_TRY(check_cache(cache, "cache"));
    if (count < 0 || count > cache->capacity)
        return fail(RIS_ERR_INVALID, "count %lld outside [0, %lld]", (long long)count, (long long)cache->capacity);
    if (first != nullptr && !aligned(first, 4)) return fail(RIS_ERR_INVALID, "first is misaligned");
    if (count == 0) return RIS_OK;
    RIS_TRY(check_ptr(k, "k"));
    RIS_TRY(check_ptr(v, "v"));
    if ((int64_t)cache->batch * cache->kv_heads * ((count + 63) / 64) > 2147483647LL) return fail(RIS_ERR_UNSUPPORTED, "too many rows for one call");
    RIS_CUDA(launch_cache4_read(cache_args(cache), first, count, k, v, reinterpret_cast<cudaStream_t>(stream)));
    return RIS_OK;
}

ris_status ris_cache4_attend(const ris_cache4 *cache, const void *q, int32_t heads, int32_t dtype, int32_t out_dtype,
                             int64_t longest, void *out, float *lse, const float *weight_in, float *weight_out, void *stream)
{
    RIS_TRY(check_cache(cache, "cache"));
    RIS_TRY(check_heads(heads, cache->kv_heads, cache->head_dim));
    RIS_TRY(check_dtype(dtype, "dtype"));
    RIS_TRY(check_dtype(out_dtype, "out_dtype"));
    RIS_TRY(check_ptr(q, "q"));
    RIS_TRY(check_ptr(out, "out"));
    if (lse != nullptr && !aligned(lse, 16)) return fail(RIS_ERR_INVALID, "lse is not 16-byte aligned");
    if ((weight_in != nullptr && !aligned(weight_in, 16)) || (weight_out != nullptr && !aligned(weight_out, 16)))
        return fail(RIS_ERR_INVALID, "weight_in or weight_out is not 16-byte aligned");
    if (weight_in != nullptr && weight_out == nullptr) return fail(RIS_ERR_INVALID, "weight_in without weight_out");
    if (longest < 0 || longest > cache->capacity)
        return fail(RIS_ERR_INVALID, "longest %lld outside [0, %lld]", (long long)longest, (long long)cache->capacity);
    if (weight_out != nullptr && heads / cache->kv_heads > 4096)
        return fail(RIS_ERR_UNSUPPORTED, "weights over %d query heads of a KV head (4096 at most)", heads / cache->kv_heads);
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    Cache4AttendArgs a{};
    a.c = cache_args(cache);
    a.q = q;
    a.out = out;
    a.lse = lse;
    a.weight_in = weight_in;
    a.weight_out = weight_out;
    a.Hq = heads;
    a.G = heads / cache->kv_heads;
    a.scale_log2 = (float)log2e_over_sqrt(cache->head_dim);
    a.reach = longest > 0 ? longest : cache->capacity;
    constexpr int32_t block = 8;
    const int64_t lists = (int64_t)cache->batch * cache->kv_heads * ((a.G + block - 1) / block);
    if (lists > (int64_t(1) << 24)) return fail(RIS_ERR_UNSUPPORTED, "batch x kv_heads = %lld lists", (long long)lists);
    a.lists = (int32_t)lists;
    // as many CTAs as are resident at once (cache4.cu's launch bounds), fewer where there are not as many units
    constexpr int per_sm = 3;
    a.ctas = (int32_t)std::min<int64_t>(152 * per_sm, lists * ((a.reach + kCacheUnit - 1) / kCacheUnit));
    const size_t parts = ((size_t)a.ctas + (size_t)lists) * block;
    const size_t o_b = room(sizeof(float) * parts * cache->head_dim), ml_b = room(sizeof(float2) * parts);
    a.score_pitch = (a.reach + 3) & ~int64_t(3);
    const size_t score_b = weight_out != nullptr ? sizeof(float) * (size_t)cache->batch * heads * a.score_pitch : 0;
    Scratch mem;
    const size_t list_b = room(2 * sizeof(int32_t) * (size_t)lists);
    RIS_CUDA(mem.alloc(o_b + ml_b + list_b + score_b, s));
    a.part_o = static_cast<float *>(mem.p);
    a.part_ml = reinterpret_cast<float2 *>(static_cast<char *>(mem.p) + o_b);
    a.list_cta = reinterpret_cast<int32_t *>(static_cast<char *>(mem.p) + o_b + ml_b);
    if (weight_out != nullptr) a.scores = reinterpret_cast<float *>(static_cast<char *>(mem.p) + o_b + ml_b + list_b);
    a.wait_limit = debug_wait_limit();
    a.debug_no_loads = debug_no_loads();
    RIS_CUDA(launch_cache4_attend(a, dtype, out_dtype, s));
    return RIS_OK;
}

ris_status ris_cache4_evict(const ris_cache4 *src, const ris_cache4 *dst, int32_t budget, int32_t recent, int32_t *kept,
                            void *stream)
{
    RIS_TRY(check_cache(src, "src"));
    RIS_TRY(check_cache(dst, "dst"));
    if (src->batch != dst->batch || src->kv_heads != dst->kv_heads || src->head_dim != dst->head_dim)
        return fail(RIS_ERR_INVALID, "src and dst differ in batch, kv_heads or head_dim");
    if (budget < 1 || budget > dst->capacity)
        return fail(RIS_ERR_INVALID, "budget %d outside [1, %lld], the target's capacity", budget, (long long)dst->capacity);
    if (recent < 0 || recent >= budget) return fail(RIS_ERR_INVALID, "recent %d outside [0, budget)", recent);
    RIS_TRY(check_ptr(kept, "kept"));
    const bool same = src->k == dst->k;
    const void *const x[] = {src->v, src->k_scale, src->v_scale, src->pos, src->weight, src->length};
    const void *const y[] = {dst->v, dst->k_scale, dst->v_scale, dst->pos, dst->weight, dst->length};
    for (int i = 0; i < 6; ++i)
        if ((x[i] == y[i]) != same) return fail(RIS_ERR_INVALID, "src and dst share some of their arrays");
    if (same && src->capacity != dst->capacity) return fail(RIS_ERR_INVALID, "in place, but the capacities differ");
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    const int64_t lists = (int64_t)src->batch * src->kv_heads;
    if (lists > (int64_t(1) << 24) || lists * (budget / 64 + 1) > 2147483647LL)
        return fail(RIS_ERR_UNSUPPORTED, "batch x kv_heads = %lld lists of %d slots", (long long)lists, budget);
    Cache4EvictArgs a{};
    a.src = cache_args(src);
    a.dst = cache_args(dst);
    a.in_place = same;
    a.budget = budget;
    a.recent = recent;
    a.kept = kept;
    Scratch holes;
    RIS_CUDA(holes.alloc(sizeof(int32_t) * (size_t)src->batch * src->kv_heads * budget, s));
    RIS_CUDA(launch_cache4_evict(a, static_cast<int32_t *>(holes.p), s));
    return RIS_OK;
}

// ---------------------------------------------------------------- normed and turned heads
ris_status ris_norm_rope(const void *q, const void *k, void *q_out, void *k_out, int32_t dtype, int64_t n, int32_t heads,
                         int32_t kv_heads, int32_t head_dim, int64_t q_stride, int64_t k_stride, int64_t q_out_stride,
                         int64_t k_out_stride, const int32_t *positions, const void *q_weight, const void *k_weight, float eps,
                         int32_t rot_dim, int32_t pairs, int64_t n_ctx, const ris_rope_cfg *rope, void *stream)
{
    NormRopeArgs a{};
    RIS_TRY(norm_rope_args(a, dtype, n, heads, kv_heads, head_dim, positions, q_weight, k_weight, eps, rot_dim, pairs, n_ctx, rope));
    if (n == 0) return RIS_OK;
    const void *const x[] = {q, k};
    void *const y[] = {q_out, k_out};
    const int64_t xs[] = {q_stride, k_stride}, ys[] = {q_out_stride, k_out_stride};
    static const char *const name[2][4] = {{"q", "q_out", "q_stride", "q_out_stride"}, {"k", "k_out", "k_stride", "k_out_stride"}};
    for (int w = 0; w < (kv_heads > 0 ? 2 : 1); ++w) {
        RIS_TRY(check_ptr(x[w], name[w][0]));
        RIS_TRY(check_ptr(y[w], name[w][1]));
        RIS_TRY(check_stride(xs[w], (int64_t)a.heads[w] * head_dim, dtype, name[w][2]));
        RIS_TRY(check_stride(ys[w], (int64_t)a.heads[w] * head_dim, dtype, name[w][3]));
        if (x[w] == y[w] && xs[w] != ys[w]) return fail(RIS_ERR_INVALID, "%s in place with another stride", name[w][0]);
        a.x[w] = x[w], a.y[w] = y[w];
        a.x_stride[w] = xs[w], a.y_stride[w] = ys[w];
    }
    RIS_CUDA(launch_norm_rope(a, dtype, head_dim, pairs != 0, reinterpret_cast<cudaStream_t>(stream)));
    return RIS_OK;
}

ris_status ris_norm_rope_backward(const void *dq, const void *dk, const void *q, const void *k, void *gq, void *gk, float *gq_weight,
                                  float *gk_weight, int32_t dtype, int64_t n, int32_t heads, int32_t kv_heads, int32_t head_dim,
                                  int64_t dq_stride, int64_t dk_stride, int64_t q_stride, int64_t k_stride, int64_t gq_stride,
                                  int64_t gk_stride, const int32_t *positions, const void *q_weight, const void *k_weight, float eps,
                                  int32_t rot_dim, int32_t pairs, int64_t n_ctx, const ris_rope_cfg *rope, void *stream)
{
    NormRopeArgs a{};
    RIS_TRY(norm_rope_args(a, dtype, n, heads, kv_heads, head_dim, positions, q_weight, k_weight, eps, rot_dim, pairs, n_ctx, rope));
    float *const gw[] = {gq_weight, gk_weight};
    for (int w = 0; w < 2; ++w) {
        if ((gw[w] != nullptr) != (a.weight[w] != nullptr)) return fail(RIS_ERR_INVALID, "a weight's gradient is wanted for each weight, and for no other");
        if (gw[w] != nullptr && !aligned(gw[w], 4)) return fail(RIS_ERR_INVALID, "a weight's gradient is misaligned");
    }
    const void *const dy[] = {dq, dk}, *const x[] = {q, k};
    void *const y[] = {gq, gk};
    const int64_t ds[] = {dq_stride, dk_stride}, xs[] = {q_stride, k_stride}, ys[] = {gq_stride, gk_stride};
    static const char *const name[2][6] = {{"dq", "q", "gq", "dq_stride", "q_stride", "gq_stride"}, {"dk", "k", "gk", "dk_stride", "k_stride", "gk_stride"}};
    for (int w = 0; n > 0 && w < (kv_heads > 0 ? 2 : 1); ++w) {
        const int64_t row = (int64_t)a.heads[w] * head_dim;
        RIS_TRY(check_ptr(dy[w], name[w][0]));
        RIS_TRY(check_ptr(y[w], name[w][2]));
        RIS_TRY(check_stride(ds[w], row, dtype, name[w][3]));
        RIS_TRY(check_stride(ys[w], row, dtype, name[w][5]));
        if (dy[w] == y[w] && ds[w] != ys[w]) return fail(RIS_ERR_INVALID, "%s in place with another stride", name[w][0]);
        if (a.weight[w] != nullptr) {  // (the rotation alone does not ask for its inputs)
            RIS_TRY(check_ptr(x[w], name[w][1]));
            RIS_TRY(check_stride(xs[w], row, dtype, name[w][4]));
            if (x[w] == y[w] && xs[w] != ys[w]) return fail(RIS_ERR_INVALID, "%s in place with another stride", name[w][1]);
        }
        a.dy[w] = dy[w], a.x[w] = x[w], a.y[w] = y[w];
        a.dy_stride[w] = ds[w], a.x_stride[w] = xs[w], a.y_stride[w] = ys[w];
    }
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    norm_rope_ctas(dtype, head_dim, n, a.heads, a.ctas);
    Scratch mem;
    if (n > 0 && (gq_weight != nullptr || gk_weight != nullptr)) {
        RIS_CUDA(mem.alloc(sizeof(float2) * (size_t)(a.ctas[0] + a.ctas[1]) * head_dim, s));
        a.part = static_cast<float2 *>(mem.p);
    }
    if (n > 0 || gq_weight != nullptr || gk_weight != nullptr) RIS_CUDA(launch_norm_rope_backward(a, dtype, head_dim, pairs != 0, gq_weight, gk_weight, s));
    return RIS_OK;
}

// ---------------------------------------------------------------- the cache in pages
ris_status ris_paged_append(const ris_paged *cache, ris_pack_t pack, const void *k, const void *v, int64_t k_stride, int64_t v_stride,
                            const int32_t *start, void *stream)
{
    RIS_TRY(check_paged(cache));
    if (pack == nullptr) return fail(RIS_ERR_INVALID, "pack is NULL");
    if (pack->n_seqs != cache->batch)
        return fail(RIS_ERR_INVALID, "the pack has %d sequences, the cache %d", pack->n_seqs, cache->batch);
    if (start != nullptr && (!aligned(start, 4) || start == cache->length))
        return fail(RIS_ERR_INVALID, "start is misaligned or the cache's own lengths (pass NULL for those)");
    if (pack->q_total > 0) {
        RIS_TRY(check_ptr(k, "k"));
        RIS_TRY(check_ptr(v, "v"));
        RIS_TRY(check_stride(k_stride, (int64_t)cache->kv_heads * cache->head_dim, cache->dtype, "k_stride"));
        RIS_TRY(check_stride(v_stride, (int64_t)cache->kv_heads * cache->head_dim, cache->dtype, "v_stride"));
    }
    PagedAppendArgs a{};
    a.c = paged_args(cache);
    a.k = k, a.v = v;
    a.k_stride = k_stride, a.v_stride = v_stride;
    a.start = start;
    a.off = pack->q_off;
    a.seq_of = pack->seq_of;
    a.total = pack->q_total;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    const PackUse use{pack, s};
    RIS_CUDA(launch_paged_append(a, cache->dtype, s));
    return RIS_OK;
}

ris_status ris_paged_attend(const ris_paged *cache, ris_pack_t pack, const void *q, int64_t q_stride, int32_t heads, int32_t window,
                            int32_t anchors, int64_t longest, void *out, float *lse, void *stream)
{
    RIS_TRY(check_paged(cache));
    if (pack == nullptr) return fail(RIS_ERR_INVALID, "pack is NULL");
    if (pack->n_seqs != cache->batch)
        return fail(RIS_ERR_INVALID, "the pack has %d sequences, the cache %d", pack->n_seqs, cache->batch);
    RIS_TRY(check_heads(heads, cache->kv_heads, cache->head_dim));
    if (window < 0 || anchors < 0) return fail(RIS_ERR_INVALID, "window and anchors must be >= 0");
    if (window == 0 && anchors != 0) return fail(RIS_ERR_INVALID, "anchors without a window");
    const int64_t capacity = (int64_t)cache->table_len * cache->page_size;
    if (longest < 0 || longest > capacity) return fail(RIS_ERR_INVALID, "longest %lld outside [0, %lld]", (long long)longest, (long long)capacity);
    if (lse != nullptr && !aligned(lse, 16)) return fail(RIS_ERR_INVALID, "lse is not 16-byte aligned");
    if (pack->q_total == 0) return RIS_OK;
    RIS_TRY(check_ptr(q, "q"));
    RIS_TRY(check_ptr(out, "out"));
    RIS_TRY(check_stride(q_stride, (int64_t)heads * cache->head_dim, cache->dtype, "q_stride"));
    {  // (a second pass reads the queries again, after outputs have been written)
        const uintptr_t row = (uintptr_t)heads * cache->head_dim, esz = cache->dtype == RIS_F32 ? 4 : 2, n = (uintptr_t)pack->q_total;
        const uintptr_t q0 = reinterpret_cast<uintptr_t>(q), o0 = reinterpret_cast<uintptr_t>(out);
        if (q0 < o0 + n * row * esz && o0 < q0 + ((n - 1) * (uintptr_t)q_stride + row) * esz) return fail(RIS_ERR_INVALID, "out overlaps q");
    }
    PagedAttendArgs a{};
    a.c = paged_args(cache);
    a.q = q;
    a.out = out;
    a.lse = lse;
    a.q_stride = q_stride;
    a.q_total = pack->q_total;
    a.off = pack->q_off;
    a.Hq = heads;
    a.G = heads / cache->kv_heads;
    a.window = std::min(window, 1 << 30);  // (no sequence is longer)
    a.anchors = std::min(anchors, 1 << 30);
    a.reach = (int32_t)(longest > 0 ? longest : capacity);
    a.scale_log2 = (float)log2e_over_sqrt(cache->head_dim);
    a.wait_limit = debug_wait_limit() > 0 ? debug_wait_limit() : int64_t(1) << 31;
    a.debug_no_loads = debug_no_loads();
    const bool tiles = cache->dtype == RIS_BF16;
    a.unit_cost = paged_unit_cost(tiles, cache->head_dim);
    const int32_t tile_rows = tiles ? kPagedTileRows : paged_f32_rows((int64_t)pack->q_longest * a.G);
    a.block = std::min(a.G, tile_rows);
    a.blocks = (a.G + a.block - 1) / a.block;
    a.tokens = tile_rows / a.block;
    a.part_rows = (int32_t)std::min<int64_t>(a.tokens, pack->q_longest) * a.block;
    const int32_t keys = tiles ? kPagedTileKeys : kPagedF32Keys;  // of a tile
    const int32_t places = kPagedSMs * (tiles ? paged_tile_ctas(cache->head_dim) : 2);  // of CTAs
    const int64_t items = pack->q_longest <= a.tokens ? pack->n_seqs : pack->q_total / a.tokens + pack->n_seqs;
    if (pack->q_longest > a.tokens) a.max_items = (int32_t)items;
    // no more CTAs than the longest line there can be has key tiles
    const int64_t most = a.reach / keys + 2 + a.unit_cost, line = items * cache->kv_heads * a.blocks;
    a.line = line;
    a.runs = (int32_t)std::min<int64_t>(places, line > places ? line : line * most);
    const bool plan = a.max_items > 0;
    const size_t prefix_b = plan ? room(sizeof(int64_t) * (items + 1)) : 0, item_b = plan ? room(sizeof(PagedItem) * items) : 0,
                 seq_b = plan ? room(sizeof(int32_t) * (pack->n_seqs + 1)) : 0, split_b = room(sizeof(PagedSplit) * a.runs),
                 ml_b = room(sizeof(float4) * 2 * a.runs * a.part_rows), o_b = room(sizeof(float) * 2 * a.runs * a.part_rows * cache->head_dim);
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    const PackUse use{pack, s};
    Scratch mem;
    RIS_CUDA(mem.alloc(prefix_b + item_b + seq_b + split_b + ml_b + o_b, s));
    char *d = static_cast<char *>(mem.p);
    a.prefix = reinterpret_cast<int64_t *>(d), d += prefix_b;
    a.items = reinterpret_cast<PagedItem *>(d), d += item_b;
    a.n_items = reinterpret_cast<int32_t *>(d), a.seq_items = a.n_items + 1, d += seq_b;
    a.split = reinterpret_cast<PagedSplit *>(d), d += split_b;
    a.part_ml = reinterpret_cast<float4 *>(d), d += ml_b;
    a.part_o = reinterpret_cast<float *>(d);
    if (plan) RIS_CUDA(launch_paged_plan(a, cache->dtype, s));
    RIS_CUDA(tiles ? launch_paged_tiles(a, s) : launch_paged_f32(a, tile_rows, s));
    if (a.runs > 1) RIS_CUDA(launch_paged_join(a, cache->dtype, s));
    return RIS_OK;
}

}  // extern "C"
