// Declarations shared by the executor's host side and its kernels.  The operations are specified in include/infaas_sel.h.
#pragma once

#include "infaas_sel.h"

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace infaas {

// ---- types ------------------------------------------------------------------------------------

typedef __bf16 bf16_t;
typedef _Float16 fp16_t;
template <typename T, int N> using vec = T __attribute__((ext_vector_type(N)));

// ---- attention: the plan ----------------------------------------------------------------------

// The rows of a tile are the (token, query head) pairs of whole tokens for one KV head, token-major.
constexpr int kTileRows = 128;
// Items that a plan aims at.  Tiles of many rows wait for their products: two items to each of the two workgroups that a
// compute unit holds, so that the end of a launch is a quarter of a workgroup's time at most.  Tiles of few rows wait for
// memory, whose rate those that are left share: one item to each, with the fewest starts and the least to merge.  (1024, so
// 512: prompts behind 16k keys 925 us, so 943; one sequence of 131k keys 122, so 116; 256 sequences behind 32k 448, so 414.
// In between, with a part of the workgroups going twice, prompts took 1447 at 640.)
constexpr int kTargetItems = 1024, kFewItems = 512;
constexpr int kFewRows = kTileRows / 2;
// Keys of an item, at least: a tile.  (Four sequences of 700 keys: 15.8 us with 256, 13.5 with 128, 12.2 with 64.)
constexpr int kMinChunk = 64;
constexpr int kChunkStep = 64;

// Keys of a sequence, at most: the loops over tiles count in 32 bits, and look the rows of two tiles and 112 keys more up ahead.
constexpr int64_t kMostKeys = INT32_MAX - 255;

constexpr int kDies = 8;             // workgroups go to the dies in turn, each with an L2 of its own
// What an item costs besides its keys (queries, first loads, results), in keys.
constexpr int kItemCost = 128;

struct PlanHeader {
    uint32_t magic;
    int32_t num_tokens, num_seqs, num_groups, heads, kv_heads, head_dim;
    int32_t max_len, table_width, page_shift;
    int32_t num_items;               // over all KV heads
    int32_t rows;                    // partial rows of one KV head
    int32_t die_start[2][kDies + 1]; // items of each die, of groups and of sequences: stretches of equal cost
    int32_t pad[2];
};
static_assert(sizeof(PlanHeader) == 128, "");
constexpr uint32_t kPlanMagic = 0x1f5e9a7du;

// One workgroup's work: the tokens t0 .. t0+nt-1 for one KV head and the keys k0 .. k1-1 in the pages of one sequence.
struct PlanItem {
    int32_t t0, nt, k0, k1, seq, head;
    int32_t base;                    // partial row of the first token's first head, or -1: the result is final
    int32_t pad;
};

// Where a token's partial results are: `splits` rows, `stride` apart, the first at `base` (+ query head within the KV
// head, + KV head * PlanHeader::rows).  Keys below `limit` are seen.
struct PlanToken {
    int32_t own_base, own_splits, own_stride;
    int32_t pre_base, pre_splits, pre_stride;
    int32_t limit;
    int32_t direct;                  // the result is written by the only item there is
};

// Groups, then sequences, as the plan divides them: the longest items come first.
struct PlanUnit {
    int64_t first_cost;              // of what is in front of it, of one KV head
    int32_t first_item, first_row;   // the same
    int32_t splits, tiles;
    int64_t cost;                    // of one of its items
};

struct PlanSizes {
    int64_t tokens_at, units_at, items_at, bytes;
    int64_t max_items, max_rows;     // items over all KV heads; partial rows of one KV head
};

struct PlanView {
    PlanHeader *head;
    PlanToken *tokens;
    PlanUnit *units;
    PlanItem *items;
};

// ---- arguments of the kernels -----------------------------------------------------------------

struct CacheArgs {
    void *k, *v;
    const int32_t *table;
    int64_t num_pages, page_stride, slot_stride, head_stride;
    int32_t table_width, page_shift, max_len;
};

struct BatchArgs {
    int32_t num_tokens, num_seqs, num_groups, heads, kv_heads, head_dim;
    const int32_t *token_seq, *token_pos, *seq_start, *seq_len, *group_start, *shared_len;
};

struct AttendArgs {
    BatchArgs batch;
    CacheArgs cache;
    PlanView plan;
    const void *q;
    void *out;
    int64_t q_token_stride, q_head_stride, out_token_stride, out_head_stride;
    float scale_log2;                // scale * log2(e)
    float *part_o;                   // [rows][head_dim]
    float2 *part_ml;                 // [rows] reference of the weights (of scores in units of log 2) and their sum
};

struct AppendArgs {
    infaas_sel_append_args a;
    CacheArgs cache;
    const int32_t *token_seq, *token_pos;
    int32_t num_tokens, num_seqs, heads, kv_heads, head_dim;
};

struct SampleArgs {
    const void *logits;
    int64_t row_stride;
    int32_t rows, vocab;
    const float *temperature, *top_p, *min_p, *draw;
    const int32_t *top_k;
    int32_t *token;
    float *prob;
};

// Workgroups of a launch, at most: a grid of 2^32 threads and more is cut to its low 32 bits without an error.
constexpr int64_t kMostGroups = 1 << 16;

hipError_t launch_plan(const BatchArgs &b, const CacheArgs &c, const PlanView &p, const PlanSizes &z, hipStream_t s);
hipError_t launch_attend(const AttendArgs &a, int32_t type, int64_t max_items, hipStream_t s);
hipError_t launch_append(const AppendArgs &a, int32_t type, hipStream_t s);
hipError_t launch_sample(const SampleArgs &a, int32_t type, hipStream_t s);

}  // namespace infaas
