// Host side of the executor: handle, checks of arguments, scratch memory, launches.
// The calls are specified in include/infaas_sel.h.
#include "exec.h"
#include "internal.h"

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <new>
#include <vector>

using namespace infaas;

struct infaas_sel_exec {
    int32_t device = 0;
    void *scratch = nullptr;
    int64_t scratch_bytes = 0;
    std::vector<void *> retired;   // smaller scratch blocks: graphs recorded with them may still be replayed
};

namespace {

int refuse(const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(error_text(), kErrorText, fmt, ap);
    va_end(ap);
    return INFAAS_SEL_ERR_INVALID_ARG;
}

int hip_failed(hipError_t e, const char *what)
{
    snprintf(error_text(), kErrorText, "%s: %s (%d)", what, hipGetErrorString(e), (int)e);
    (void)hipGetLastError();
    return INFAAS_SEL_ERR_HIP;
}

struct OnDevice {
    int prev = -1, target;
    hipError_t err;
    explicit OnDevice(int dev) : target(dev)
    {
        err = hipGetDevice(&prev);
        if (err == hipSuccess && prev != dev) err = hipSetDevice(dev);
    }
    ~OnDevice()
    {
        if (prev >= 0 && prev != target) (void)hipSetDevice(prev);
    }
};

bool aligned(const void *p) { return ((uintptr_t)p & 15) == 0; }
bool vector_stride(int64_t s) { return s % 8 == 0; }

int check_cache(const infaas_sel_cache *c)
{
    if (!c) return refuse("cache: null");
    if (c->type != INFAAS_SEL_TYPE_BF16 && c->type != INFAAS_SEL_TYPE_FP16) return refuse("cache: type %d", c->type);
    if (c->kv_heads < 1 || c->kv_heads > 65536) return refuse("cache: %d KV heads", c->kv_heads);
    if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256)
        return refuse("cache: head dimension %d is not 64, 128 or 256", c->head_dim);
    if (c->page_size < 1 || c->page_size > 65536 || (c->page_size & (c->page_size - 1)))
        return refuse("cache: page size %d is not a power of two up to 65536", c->page_size);
    return INFAAS_SEL_OK;
}

int check_pools(const infaas_sel_cache *c)
{
    if (!c->d_k || !c->d_v || !aligned(c->d_k) || !aligned(c->d_v)) return refuse("cache: pools are null or not aligned to 16 bytes");
    if (c->num_pages < 1) return refuse("cache: %lld pages", (long long)c->num_pages);
    if (!vector_stride(c->page_stride) || !vector_stride(c->slot_stride) || !vector_stride(c->head_stride))
        return refuse("cache: strides are not multiples of 8 elements");
    if (c->page_stride < 0 || c->slot_stride < 0 || c->head_stride < 0) return refuse("cache: a negative stride");
    return INFAAS_SEL_OK;
}

int check_scales(const infaas_sel_cache *c, const infaas_sel_scales *s)
{
    if (!s) return refuse("scales: null");
    if (!s->d_k_scale || !s->d_v_scale) return refuse("scales: null arrays");
    if (s->block < 1 || s->block > c->page_size || (s->block & (s->block - 1)))
        return refuse("scales: a block of %d keys is not a power of two up to the page size %d", s->block, c->page_size);
    if (s->page_stride < 0 || s->block_stride < 0 || s->head_stride < 0) return refuse("scales: a negative stride");
    if (c->page_stride % 16 || c->slot_stride % 16 || c->head_stride % 16)
        return refuse("cache: strides of codes are not multiples of 16");
    return INFAAS_SEL_OK;
}

// Sizes that the batch and the cache have to agree on; looks at no pointer.
int check_sizes(const infaas_sel_cache *c, const infaas_sel_batch *b)
{
    if (int rc = check_cache(c)) return rc;
    if (!b) return refuse("batch: null");
    if (b->num_tokens < 0 || b->num_seqs < 0 || b->num_groups < 0 || b->max_len < 0 || b->table_width < 0)
        return refuse("batch: a negative size");
    if (b->num_groups > b->num_seqs) return refuse("batch: %d groups of %d sequences", b->num_groups, b->num_seqs);
    if (b->heads < 1 || b->heads % c->kv_heads || b->heads / c->kv_heads > kTileRows)
        return refuse("batch: %d query heads on %d KV heads (a multiple, at most %d to each)", b->heads, c->kv_heads, kTileRows);
    return INFAAS_SEL_OK;
}

int check_arrays(const infaas_sel_batch *b)
{
    if (b->num_tokens > 0 && (!b->d_token_seq || !b->d_token_pos)) return refuse("batch: null token arrays");
    if (b->num_seqs > 0 && b->table_width > 0 && !b->d_page_table) return refuse("batch: null page table");
    return INFAAS_SEL_OK;
}

int check_plan_arrays(const infaas_sel_batch *b, const PlanSizes &z)
{
    if (b->num_seqs > 0 && (!b->d_seq_start || !b->d_seq_len)) return refuse("batch: null sequence arrays");
    if (b->num_groups > 0 && (!b->d_group_start || !b->d_shared_len)) return refuse("batch: null group arrays");
    if (!b->d_plan || !aligned(b->d_plan)) return refuse("batch: the plan is null or not aligned to 16 bytes");
    if (b->plan_bytes < z.bytes)
        return refuse("batch: a plan of %lld bytes where %lld are needed", (long long)b->plan_bytes, (long long)z.bytes);
    return INFAAS_SEL_OK;
}

// False when the batch is too large for 32-bit items and rows.
bool plan_sizes(const infaas_sel_cache *c, const infaas_sel_batch *b, PlanSizes *z)
{
    const int64_t n = b->num_tokens, H = c->kv_heads, G = b->heads / c->kv_heads;
    const int64_t units = (int64_t)b->num_seqs + b->num_groups, per_tile = kTileRows / G;
    // tokens are in a tile of their own and one of their group's; the division into chunks adds what was aimed at
    const int64_t tiles = 2 * (n / per_tile) + units;
    // (an item has kMinChunk keys but for the last of each tile)
    z->max_items = std::min(kTargetItems + H * (1 + tiles), H * tiles * (b->max_len / kMinChunk + 1));
    z->max_rows = (int64_t)kTileRows * (kTargetItems / H + 2) + 2 * n * G;
    z->tokens_at = sizeof(PlanHeader);
    z->units_at = z->tokens_at + n * (int64_t)sizeof(PlanToken);
    z->items_at = z->units_at + units * (int64_t)sizeof(PlanUnit);
    z->bytes = z->items_at + z->max_items * (int64_t)sizeof(PlanItem);
    return z->max_items < INT32_MAX && z->max_rows * H < INT32_MAX;
}

int64_t scratch_for(const infaas_sel_cache *c, const PlanSizes &z)
{
    return z.max_rows * c->kv_heads * (int64_t)(c->head_dim * sizeof(float) + sizeof(float2));
}

// At least `bytes` of scratch memory; `s` is the stream of the call, or null outside one.
int ensure(infaas_sel_exec *x, int64_t bytes, hipStream_t s, bool in_call, const char *reserve = "infaas_sel_exec_reserve")
{
    if (x->scratch_bytes >= bytes) return INFAAS_SEL_OK;
    if (in_call) {
        hipStreamCaptureStatus st = hipStreamCaptureStatusNone;
        if (hipError_t e = hipStreamIsCapturing(s, &st)) return hip_failed(e, "hipStreamIsCapturing");
        if (st != hipStreamCaptureStatusNone)
            return refuse("scratch memory has to grow while the stream is being captured: call %s first", reserve);
    }
    // (half as much again, so that what is retired stays below twice what is in use)
    const int64_t want = std::max(bytes, x->scratch_bytes + x->scratch_bytes / 2);
    void *p = nullptr;
    try {
        x->retired.reserve(x->retired.size() + 1);
    } catch (const std::bad_alloc &) {
        return INFAAS_SEL_ERR_OOM;
    }
    if (hipMalloc(&p, (size_t)want) != hipSuccess) {
        (void)hipGetLastError();
        return INFAAS_SEL_ERR_OOM;
    }
    if (x->scratch) x->retired.push_back(x->scratch);
    x->scratch = p;
    x->scratch_bytes = want;
    return INFAAS_SEL_OK;
}

CacheArgs cache_args(const infaas_sel_cache *c, const infaas_sel_batch *b, const infaas_sel_scales *s = nullptr)
{
    CacheArgs a{};
    a.k = c->d_k; a.v = c->d_v;
    a.table = b->d_page_table;
    a.num_pages = c->num_pages;
    a.page_stride = c->page_stride; a.slot_stride = c->slot_stride; a.head_stride = c->head_stride;
    a.table_width = b->table_width;
    a.page_shift = __builtin_ctz((unsigned)c->page_size);
    // (what the table can hold, and what the kernels can count a few tiles beyond)
    a.max_len = (int32_t)std::min<int64_t>({b->max_len, (int64_t)b->table_width * c->page_size, kMostKeys});
    if (s) {
        a.k_scale = (uint8_t *)s->d_k_scale; a.v_scale = (uint8_t *)s->d_v_scale;
        a.block_shift = __builtin_ctz((unsigned)s->block);
        a.scale_page_stride = s->page_stride; a.scale_block_stride = s->block_stride; a.scale_head_stride = s->head_stride;
    }
    return a;
}

BatchArgs batch_args(const infaas_sel_cache *c, const infaas_sel_batch *b)
{
    return BatchArgs{b->num_tokens, b->num_seqs, b->num_groups, b->heads, c->kv_heads, c->head_dim,
                     b->d_token_seq, b->d_token_pos, b->d_seq_start, b->d_seq_len, b->d_group_start, b->d_shared_len};
}

PlanView plan_view(const infaas_sel_batch *b, const PlanSizes &z)
{
    char *p = (char *)b->d_plan;
    return PlanView{(PlanHeader *)p, (PlanToken *)(p + z.tokens_at), (PlanUnit *)(p + z.units_at), (PlanItem *)(p + z.items_at)};
}

int check_beam(int32_t queries, int32_t beams, int32_t vocab, int32_t picks, int32_t type)
{
    if (queries < 0) return refuse("beam: %d queries", queries);
    if (beams < 1 || beams > kMostBeams || picks < 1 || picks > kMostBeams)
        return refuse("beam: %d beams and %d picks (1 .. %d)", beams, picks, kMostBeams);
    if (vocab < 1 || vocab > 1 << 20) return refuse("beam: a vocabulary of %d (1 .. 1048576)", vocab);
    if (type != INFAAS_SEL_TYPE_FP32 && type != INFAAS_SEL_TYPE_BF16 && type != INFAAS_SEL_TYPE_FP16) return refuse("beam: type %d", type);
    // (a part of a row has 2048 logits at least)
    if ((int64_t)queries * beams * (vocab / 2048 + 1) > INT32_MAX) return refuse("beam: %d queries of %d beams", queries, beams);
    return INFAAS_SEL_OK;
}

int check_table(const infaas_sel_table *t)
{
    if (!t) return refuse("table: null");
    if (t->num_seqs < 1 || t->num_seqs > kMostSeqs) return refuse("table: %d sequences (1 .. %d)", t->num_seqs, kMostSeqs);
    if (t->table_width < 1 || t->num_pages < 1 || t->max_tokens < 1)
        return refuse("table: %d pages to a row, %d pages, %d tokens (1 at least)", t->table_width, t->num_pages, t->max_tokens);
    if (t->page_size < 1 || t->page_size > 65536 || (t->page_size & (t->page_size - 1)))
        return refuse("table: page size %d is not a power of two up to 65536", t->page_size);
    if (!t->d_page_table || !t->d_seq_len || !t->d_page_refs || !t->d_seq_start || !t->d_token_seq || !t->d_token_pos || !t->d_taken ||
        !t->d_copies)
        return refuse("table: null arrays");
    if (!aligned(t->d_page_refs)) return refuse("table: the pages' counts are not aligned to 16 bytes");
    return INFAAS_SEL_OK;
}

// infaas_sel_exec_append, and _append_scaled where `coded`.
int append(infaas_sel_exec *x, const infaas_sel_cache *cache, const infaas_sel_scales *scales, bool coded, const infaas_sel_batch *batch,
           const infaas_sel_append_args *args, void *hip_stream)
{
    if (!x) return refuse("executor: null");
    if (int rc = check_sizes(cache, batch)) return rc;
    if (int rc = check_pools(cache)) return rc;
    if (coded)
        if (int rc = check_scales(cache, scales)) return rc;
    if (int rc = check_arrays(batch)) return rc;
    if (coded && batch->num_seqs > 0 && !batch->d_seq_start) return refuse("batch: null sequence arrays");
    if (!args) return refuse("append: null");
    if (args->rot_dim < 0 || args->rot_dim > cache->head_dim || args->rot_dim % 16)
        return refuse("append: %d rotated dimensions (a multiple of 16 up to %d)", args->rot_dim, cache->head_dim);
    if (args->rot_dim > 0 && !args->d_freq) return refuse("append: null frequencies");
    if ((args->d_q == nullptr) != (args->d_q_out == nullptr)) return refuse("append: queries without an output, or the reverse");
    if (batch->num_tokens == 0) return INFAAS_SEL_OK;
    if (!args->d_k || !args->d_v || !aligned(args->d_k) || !aligned(args->d_v) || !aligned(args->d_q) || !aligned(args->d_q_out))
        return refuse("append: arrays are null or not aligned to 16 bytes");
    for (int64_t s : {args->q_token_stride, args->q_head_stride, args->k_token_stride, args->k_head_stride, args->v_token_stride,
                      args->v_head_stride, args->out_token_stride, args->out_head_stride})
        if (!vector_stride(s)) return refuse("append: strides are not multiples of 8 elements");
    OnDevice on(x->device);
    if (on.err != hipSuccess) return hip_failed(on.err, "hipSetDevice");
    AppendArgs a{*args, cache_args(cache, batch, scales), batch->d_token_seq, batch->d_token_pos, batch->num_tokens, batch->num_seqs,
                 batch->heads, cache->kv_heads, cache->head_dim};
    if (coded) {
        const AppendScaledArgs sa{a, batch->d_seq_start, 0, 0, 0, 0, 0};
        if (hipError_t e = launch_append_scaled(sa, cache->type, (hipStream_t)hip_stream)) return hip_failed(e, "infaas_sel_exec_append_scaled");
        return INFAAS_SEL_OK;
    }
    if (hipError_t e = launch_append(a, cache->type, (hipStream_t)hip_stream)) return hip_failed(e, "infaas_sel_exec_append");
    return INFAAS_SEL_OK;
}

// infaas_sel_exec_attend, and _attend_scaled where `coded`.
int attend(infaas_sel_exec *x, const infaas_sel_cache *cache, const infaas_sel_scales *scales, bool coded, const infaas_sel_batch *batch,
           const void *d_q, int64_t q_token_stride, int64_t q_head_stride,
           void *d_out, int64_t out_token_stride, int64_t out_head_stride, float scale, void *hip_stream)
{
    if (!x) return refuse("executor: null");
    if (int rc = check_sizes(cache, batch)) return rc;
    if (int rc = check_pools(cache)) return rc;
    if (coded)
        if (int rc = check_scales(cache, scales)) return rc;
    if (int rc = check_arrays(batch)) return rc;
    PlanSizes z;
    if (!plan_sizes(cache, batch, &z)) return refuse("batch: too many tokens");
    if (int rc = check_plan_arrays(batch, z)) return rc;
    if (!(scale > 0) || !std::isfinite(scale)) return refuse("attend: the scale is not finite and positive");
    if (batch->num_tokens == 0) return INFAAS_SEL_OK;
    if (!d_q || !d_out || !aligned(d_q) || !aligned(d_out)) return refuse("attend: arrays are null or not aligned to 16 bytes");
    for (int64_t s : {q_token_stride, q_head_stride, out_token_stride, out_head_stride})
        if (!vector_stride(s)) return refuse("attend: strides are not multiples of 8 elements");
    OnDevice on(x->device);
    if (on.err != hipSuccess) return hip_failed(on.err, "hipSetDevice");
    if (int rc = ensure(x, scratch_for(cache, z), (hipStream_t)hip_stream, true)) return rc;
    AttendArgs a{};
    a.batch = batch_args(cache, batch);
    a.cache = cache_args(cache, batch, scales);
    a.plan = plan_view(batch, z);
    a.q = d_q; a.out = d_out;
    a.q_token_stride = q_token_stride; a.q_head_stride = q_head_stride;
    a.out_token_stride = out_token_stride; a.out_head_stride = out_head_stride;
    a.scale_log2 = scale * 1.44269504088896f;
    a.part_o = (float *)x->scratch;
    a.part_ml = (float2 *)((char *)x->scratch + z.max_rows * cache->kv_heads * cache->head_dim * (int64_t)sizeof(float));
    if (hipError_t e = launch_attend(a, cache->type, z.max_items, (hipStream_t)hip_stream)) return hip_failed(e, coded ? "infaas_sel_exec_attend_scaled" : "infaas_sel_exec_attend");
    return INFAAS_SEL_OK;
}

}  // namespace

extern "C" {

int infaas_sel_exec_create(int32_t device, infaas_sel_exec_t **out)
{
    if (!out) return refuse("infaas_sel_exec_create: null");
    if (device < 0) return refuse("infaas_sel_exec_create: device %d", device);
    infaas_sel_exec *x = new (std::nothrow) infaas_sel_exec;
    if (!x) return INFAAS_SEL_ERR_OOM;
    x->device = device;
    *out = x;
    return INFAAS_SEL_OK;
}

void infaas_sel_exec_destroy(infaas_sel_exec_t *x)
{
    if (!x) return;
    if (x->scratch) {
        OnDevice on(x->device);
        if (on.err == hipSuccess) {
            (void)hipFree(x->scratch);   // (waits for the device)
            for (void *p : x->retired) (void)hipFree(p);
        }
    }
    delete x;
}

int64_t infaas_sel_exec_plan_bytes(const infaas_sel_cache *cache, const infaas_sel_batch *batch)
{
    PlanSizes z;
    if (check_sizes(cache, batch) != INFAAS_SEL_OK) return 0;
    if (!plan_sizes(cache, batch, &z)) { refuse("batch: too many tokens"); return 0; }
    return z.bytes;
}

int infaas_sel_exec_reserve(infaas_sel_exec_t *x, const infaas_sel_cache *cache, const infaas_sel_batch *batch)
{
    if (!x) return refuse("executor: null");
    if (int rc = check_sizes(cache, batch)) return rc;
    PlanSizes z;
    if (!plan_sizes(cache, batch, &z)) return refuse("batch: too many tokens");
    OnDevice on(x->device);
    if (on.err != hipSuccess) return hip_failed(on.err, "hipSetDevice");
    return ensure(x, scratch_for(cache, z), nullptr, false);
}

int infaas_sel_exec_plan(infaas_sel_exec_t *x, const infaas_sel_cache *cache, const infaas_sel_batch *batch, void *hip_stream)
{
    if (!x) return refuse("executor: null");
    if (int rc = check_sizes(cache, batch)) return rc;
    if (int rc = check_arrays(batch)) return rc;
    PlanSizes z;
    if (!plan_sizes(cache, batch, &z)) return refuse("batch: too many tokens");
    if (int rc = check_plan_arrays(batch, z)) return rc;
    if (batch->num_tokens == 0) return INFAAS_SEL_OK;
    OnDevice on(x->device);
    if (on.err != hipSuccess) return hip_failed(on.err, "hipSetDevice");
    if (hipError_t e = launch_plan(batch_args(cache, batch), cache_args(cache, batch), plan_view(batch, z), z, (hipStream_t)hip_stream))
        return hip_failed(e, "infaas_sel_exec_plan");
    return INFAAS_SEL_OK;
}

int infaas_sel_exec_append(infaas_sel_exec_t *x, const infaas_sel_cache *cache, const infaas_sel_batch *batch,
                           const infaas_sel_append_args *args, void *hip_stream)
{
    return append(x, cache, nullptr, false, batch, args, hip_stream);
}

int infaas_sel_exec_append_scaled(infaas_sel_exec_t *x, const infaas_sel_cache *cache, const infaas_sel_scales *scales,
                                  const infaas_sel_batch *batch, const infaas_sel_append_args *args, void *hip_stream)
{
    return append(x, cache, scales, true, batch, args, hip_stream);
}

int infaas_sel_exec_attend(infaas_sel_exec_t *x, const infaas_sel_cache *cache, const infaas_sel_batch *batch,
                           const void *d_q, int64_t q_token_stride, int64_t q_head_stride,
                           void *d_out, int64_t out_token_stride, int64_t out_head_stride, float scale, void *hip_stream)
{
    return attend(x, cache, nullptr, false, batch, d_q, q_token_stride, q_head_stride, d_out, out_token_stride, out_head_stride, scale,
                  hip_stream);
}

int infaas_sel_exec_attend_scaled(infaas_sel_exec_t *x, const infaas_sel_cache *cache, const infaas_sel_scales *scales,
                                  const infaas_sel_batch *batch, const void *d_q, int64_t q_token_stride, int64_t q_head_stride,
                                  void *d_out, int64_t out_token_stride, int64_t out_head_stride, float scale, void *hip_stream)
{
    return attend(x, cache, scales, true, batch, d_q, q_token_stride, q_head_stride, d_out, out_token_stride, out_head_stride, scale,
                  hip_stream);
}

int infaas_sel_exec_read(infaas_sel_exec_t *x, const infaas_sel_cache *cache, const infaas_sel_scales *scales,
                         const infaas_sel_batch *batch, void *d_k, int64_t k_token_stride, int64_t k_head_stride,
                         void *d_v, int64_t v_token_stride, int64_t v_head_stride, void *hip_stream)
{
    if (!x) return refuse("executor: null");
    if (int rc = check_sizes(cache, batch)) return rc;
    if (int rc = check_pools(cache)) return rc;
    if (scales)
        if (int rc = check_scales(cache, scales)) return rc;
    if (int rc = check_arrays(batch)) return rc;
    if (batch->num_tokens == 0) return INFAAS_SEL_OK;
    if (!d_k || !d_v || !aligned(d_k) || !aligned(d_v)) return refuse("read: arrays are null or not aligned to 16 bytes");
    for (int64_t s : {k_token_stride, k_head_stride, v_token_stride, v_head_stride})
        if (!vector_stride(s)) return refuse("read: strides are not multiples of 8 elements");
    OnDevice on(x->device);
    if (on.err != hipSuccess) return hip_failed(on.err, "hipSetDevice");
    const ReadArgs a{cache_args(cache, batch, scales), batch->d_token_seq, batch->d_token_pos, batch->num_tokens, batch->num_seqs,
                     cache->kv_heads, cache->head_dim, d_k, d_v, k_token_stride, k_head_stride, v_token_stride, v_head_stride};
    if (hipError_t e = launch_read(a, cache->type, (hipStream_t)hip_stream)) return hip_failed(e, "infaas_sel_exec_read");
    return INFAAS_SEL_OK;
}

int infaas_sel_exec_advance(infaas_sel_exec_t *x, const infaas_sel_table *table, const int32_t *d_new, const int32_t *d_parent,
                            void *hip_stream)
{
    if (!x) return refuse("executor: null");
    if (int rc = check_table(table)) return rc;
    if (!d_new) return refuse("advance: null arrays");
    OnDevice on(x->device);
    if (on.err != hipSuccess) return hip_failed(on.err, "hipSetDevice");
    const AdvanceArgs a{*table, d_new, d_parent, __builtin_ctz((unsigned)table->page_size),
                        (int32_t)std::min<int64_t>((int64_t)table->table_width * table->page_size, kMostKeys)};
    if (hipError_t e = launch_advance(a, (hipStream_t)hip_stream)) return hip_failed(e, "infaas_sel_exec_advance");
    return INFAAS_SEL_OK;
}

int infaas_sel_exec_copy(infaas_sel_exec_t *x, const infaas_sel_cache *cache, const infaas_sel_scales *scales,
                         const infaas_sel_table *table, void *hip_stream)
{
    if (!x) return refuse("executor: null");
    if (int rc = check_cache(cache)) return rc;
    if (int rc = check_pools(cache)) return rc;
    if (scales)
        if (int rc = check_scales(cache, scales)) return rc;
    if (int rc = check_table(table)) return rc;
    if (table->page_size != cache->page_size)
        return refuse("copy: a table for pages of %d keys with a cache's of %d", table->page_size, cache->page_size);
    OnDevice on(x->device);
    if (on.err != hipSuccess) return hip_failed(on.err, "hipSetDevice");
    infaas_sel_batch none{};
    const CopyArgs a{cache_args(cache, &none, scales), cache->kv_heads, cache->head_dim * (scales ? 1 : 2), table->num_seqs, table->d_copies};
    if (hipError_t e = launch_copy(a, (hipStream_t)hip_stream)) return hip_failed(e, "infaas_sel_exec_copy");
    return INFAAS_SEL_OK;
}

int infaas_sel_exec_sample(infaas_sel_exec_t *x, int32_t rows, int32_t vocab, int32_t type, const void *d_logits,
                           int64_t row_stride, const float *d_temperature, const int32_t *d_top_k, const float *d_top_p,
                           const float *d_min_p, const float *d_draw, int32_t *d_out_token, float *d_out_prob, void *hip_stream)
{
    if (!x) return refuse("executor: null");
    if (rows < 0) return refuse("sample: %d rows", rows);
    if (vocab < 1 || vocab > 1 << 20) return refuse("sample: a vocabulary of %d (1 .. 1048576)", vocab);
    if (type != INFAAS_SEL_TYPE_FP32 && type != INFAAS_SEL_TYPE_BF16 && type != INFAAS_SEL_TYPE_FP16) return refuse("sample: type %d", type);
    if (rows == 0) return INFAAS_SEL_OK;
    if (!d_logits || !d_draw || !d_out_token) return refuse("sample: null arrays");
    if ((uintptr_t)d_logits % (type == INFAAS_SEL_TYPE_FP32 ? 4 : 2)) return refuse("sample: logits are not aligned to their type");
    OnDevice on(x->device);
    if (on.err != hipSuccess) return hip_failed(on.err, "hipSetDevice");
    SampleArgs a{d_logits, row_stride, rows, vocab, d_temperature, d_top_p, d_min_p, d_draw, d_top_k, d_out_token, d_out_prob};
    if (hipError_t e = launch_sample(a, type, (hipStream_t)hip_stream)) return hip_failed(e, "infaas_sel_exec_sample");
    return INFAAS_SEL_OK;
}

int infaas_sel_exec_beam(infaas_sel_exec_t *x, int32_t queries, int32_t beams, int32_t vocab, int32_t picks, int32_t type,
                         const void *d_logits, int64_t row_stride, const float *d_scores, const int32_t *d_ended,
                         const float *d_factor, int32_t end_token, int32_t *d_out_parent, int32_t *d_out_token,
                         float *d_out_score, void *hip_stream)
{
    if (!x) return refuse("executor: null");
    if (int rc = check_beam(queries, beams, vocab, picks, type)) return rc;
    if (d_ended && (end_token < 0 || end_token >= vocab)) return refuse("beam: end token %d of a vocabulary of %d", end_token, vocab);
    if (queries == 0) return INFAAS_SEL_OK;
    if (!d_logits || !d_scores || !d_out_parent || !d_out_token || !d_out_score) return refuse("beam: null arrays");
    if ((uintptr_t)d_logits % (type == INFAAS_SEL_TYPE_FP32 ? 4 : 2)) return refuse("beam: logits are not aligned to their type");
    OnDevice on(x->device);
    if (on.err != hipSuccess) return hip_failed(on.err, "hipSetDevice");
    const BeamSizes z = beam_sizes(queries, beams, vocab, picks);
    if (int rc = ensure(x, z.bytes, (hipStream_t)hip_stream, true, "infaas_sel_exec_reserve_beam")) return rc;
    char *const p = (char *)x->scratch;
    const BeamArgs a{d_logits, row_stride, queries, beams, vocab, picks, end_token, (int32_t)z.chunks, (int32_t)z.parts, d_scores, d_factor, d_ended,
                     d_out_parent, d_out_token, d_out_score, (unsigned long long *)p, (double *)(p + z.sum_at), (float *)(p + z.top_at)};
    if (hipError_t e = launch_beam(a, z, type, (hipStream_t)hip_stream)) return hip_failed(e, "infaas_sel_exec_beam");
    return INFAAS_SEL_OK;
}

int infaas_sel_exec_reserve_beam(infaas_sel_exec_t *x, int32_t queries, int32_t beams, int32_t vocab, int32_t picks, int32_t type)
{
    if (!x) return refuse("executor: null");
    if (int rc = check_beam(queries, beams, vocab, picks, type)) return rc;
    OnDevice on(x->device);
    if (on.err != hipSuccess) return hip_failed(on.err, "hipSetDevice");
    return ensure(x, beam_sizes(queries, beams, vocab, picks).bytes, nullptr, false);
}

}  // extern "C"
