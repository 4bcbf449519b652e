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
    // of a cache of 8 bits (null: of 16)
    int32_t block_shift;
    uint8_t *k_scale, *v_scale;
    int64_t scale_page_stride, scale_block_stride, scale_head_stride;
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

struct AppendScaledArgs {
    AppendArgs append;
    const int32_t *seq_start;
    int32_t q_groups, q_tokens;      // workgroups for the queries, and their tokens
    int32_t chunk, shares, rows;     // tokens that one of the others looks through; how many share its columns; rows side by side
};

struct ReadArgs {
    CacheArgs cache;
    const int32_t *token_seq, *token_pos;
    int32_t num_tokens, num_seqs, kv_heads, head_dim;
    void *k, *v;
    int64_t k_token_stride, k_head_stride, v_token_stride, v_head_stride;
};

struct AdvanceArgs {
    infaas_sel_table t;
    const int32_t *more, *parent;    // d_new, d_parent
    int32_t page_shift;
    int32_t most;                    // keys that a row has room for
};

struct CopyArgs {
    CacheArgs cache;
    int32_t kv_heads, bytes;         // of a head's key
    int32_t num_seqs;
    const int32_t *copies;
};

struct BeamArgs {
    const void *logits;
    int64_t row_stride;
    int32_t queries, beams, vocab, picks, end_token, chunks, parts;
    const float *scores, *factor;
    const int32_t *ended;
    int32_t *out_parent, *out_token;
    float *out_score;
    // of every part of every row: its best (order key of the logit, ~token; 0: none), the sum of its weights, its maximum
    unsigned long long *best;
    double *sum;
    float *top;
};
struct BeamSizes { int64_t chunk, chunks, parts, sum_at, top_at, bytes; };      // a chunk's logits, a part's chunks, a row's parts
constexpr int kMostBeams = 64;       // beams, and picks

constexpr int kMostSeqs = 4096;      // of a table

struct SampleArgs {
    const void *logits;
    int64_t row_stride;
    int32_t rows, vocab;
    const float *temperature, *top_p, *min_p, *draw;
    const int32_t *top_k;
    int32_t *token;
    float *prob;
};

// ---- codes of 8 bits --------------------------------------------------------------------------

// Two of a word's four codes times 2^(e - 127), as numbers of T: one instruction, exact where T has the number (all codes with
// all scales compared with the products in 64 bits; 0 stands for 2^-127, 255 gives NaN).
template <typename T, bool UPPER> __device__ __forceinline__ vec<T, 2> decode2(uint32_t word, uint32_t e)
{
    const float scale = __uint_as_float(e << 23);
    if constexpr (sizeof(T) == 2 && __is_same(T, bf16_t)) return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(word, scale, UPPER);
    else return __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(word, scale, UPPER);
}
template <typename T> __device__ __forceinline__ vec<T, 4> decode4(uint32_t word, uint32_t e)
{
    const vec<T, 2> a = decode2<T, false>(word, e), b = decode2<T, true>(word, e);
    return vec<T, 4>{a[0], a[1], b[0], b[1]};
}
template <typename T> __device__ __forceinline__ vec<T, 8> decode8(vec<uint32_t, 2> w, uint32_t e)
{
    const vec<T, 4> a = decode4<T>(w[0], e), b = decode4<T>(w[1], e);
    return vec<T, 8>{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
}

// Four numbers as codes, rounded to the nearest, ties to even (the instruction's rounding, compared with torch's over 2^20 numbers;
// beyond 464 and for what is no number it gives NaN).
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d)
{
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}

// The page of a key, or -1.
__device__ __forceinline__ int64_t page_of(const CacheArgs &c, int seq, int num_seqs, int64_t pos)
{
    if (pos < 0 || pos >= c.max_len || (uint32_t)seq >= (uint32_t)num_seqs) return -1;
    const int64_t page = c.table[(int64_t)seq * c.table_width + (pos >> c.page_shift)];
    return page >= 0 && page < c.num_pages ? page : -1;
}

// Workgroups of a launch, at most: a grid of 2^32 threads and more is cut to its low 32 bits without an error.
constexpr int64_t kMostGroups = 1 << 16;

hipError_t launch_plan(const BatchArgs &b, const CacheArgs &c, const PlanView &p, const PlanSizes &z, hipStream_t s);
hipError_t launch_attend(const AttendArgs &a, int32_t type, int64_t max_items, hipStream_t s);
hipError_t launch_append(const AppendArgs &a, int32_t type, hipStream_t s);
hipError_t launch_append_scaled(const AppendScaledArgs &a, int32_t type, hipStream_t s);
hipError_t launch_read(const ReadArgs &a, int32_t type, hipStream_t s);
hipError_t launch_advance(const AdvanceArgs &a, hipStream_t s);
hipError_t launch_copy(const CopyArgs &a, hipStream_t s);
BeamSizes beam_sizes(int32_t queries, int32_t beams, int32_t vocab, int32_t picks);
hipError_t launch_beam(const BeamArgs &a, const BeamSizes &z, int32_t type, hipStream_t s);
hipError_t launch_sample(const SampleArgs &a, int32_t type, hipStream_t s);

}  // namespace infaas
