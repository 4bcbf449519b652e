// Attention of a ragged batch over a paged cache, what groups of sequences share read once (infaas_sel_exec_attend):
// the plan, the items and the merge of their results.
#include "exec.h"

#include <algorithm>
#include <type_traits>

namespace infaas {

namespace {

// ---- the plan ---------------------------------------------------------------------------------

constexpr int kPlanThreads = 1024;

__device__ __forceinline__ int clampi(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }

// What unit u (a group, or behind those a sequence) has to have computed: its tokens and keys.
struct UnitRange { int t0, nt, k0, k1, seq; };

__device__ __forceinline__ int seq_limit(const BatchArgs &b, const CacheArgs &c, int s) { return clampi(b.seq_len[s], 0, c.max_len); }

// Group of a sequence, or -1.
__device__ __forceinline__ int group_of(const BatchArgs &b, int s)
{
    int lo = 0, hi = b.num_groups;      // the last g with group_start[g] <= s
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (mid <= b.num_groups - 1 && b.group_start[mid] <= s) lo = mid;
        else hi = mid - 1;
    }
    return b.num_groups > 0 && b.group_start[lo] <= s && s < b.group_start[lo + 1] ? lo : -1;
}

__device__ __forceinline__ int shared_of(const BatchArgs &b, const CacheArgs &c, int g)
{
    return g < 0 ? 0 : clampi(b.shared_len[g], 0, c.max_len);
}

__device__ __forceinline__ UnitRange unit_range(const BatchArgs &b, const CacheArgs &c, int u)
{
    UnitRange r;
    if (u >= b.num_groups) {
        const int s = u - b.num_groups;
        r.seq = s;
        r.t0 = clampi(b.seq_start[s], 0, b.num_tokens);
        r.nt = clampi(b.seq_start[s + 1], r.t0, b.num_tokens) - r.t0;
        r.k1 = seq_limit(b, c, s);
        r.k0 = min(shared_of(b, c, group_of(b, s)), r.k1);
    } else {
        const int g = u;
        const int a = clampi(b.group_start[g], 0, b.num_seqs), e = clampi(b.group_start[g + 1], a, b.num_seqs);
        r.seq = a < b.num_seqs ? a : 0;
        r.t0 = clampi(b.seq_start[a], 0, b.num_tokens);
        r.nt = e > a ? clampi(b.seq_start[e], r.t0, b.num_tokens) - r.t0 : 0;
        r.k0 = 0;
        r.k1 = shared_of(b, c, g);
    }
    return r;
}

// One workgroup.  The cost of a tile is its keys; chunks are as long as would make so many items if tiles could be cut
// anywhere, and the same for all, so that items are of one length but for the last of each tile (and there are more of them:
// one at least to every tile).  How many depends on the rows of the tiles (their mean by cost): see kFewItems.
// 9 to 11 us for few sequences, 16 to 20 for 256 behind prefixes or four prompts of 2048: once a step, for all layers.
// The cost counts all keys of a sequence, also those behind a tile's tokens.  Behind a long prefix that is nothing; of a prompt
// alone the dies' work is uneven (1024 tokens of 32 heads on 8: from 2.1 to 0.02 of the mean, 45 us), below 4096
// tokens, from which on a tile is one item.
__global__ __launch_bounds__(kPlanThreads) void k_plan(BatchArgs b, CacheArgs c, PlanView p, int max_items, int max_rows)
{
    __shared__ unsigned long long cost, row_cost;
    __shared__ long long scan[3][kPlanThreads / 64];
    __shared__ long long totals[3];
    const int tid = threadIdx.x, G = b.heads / b.kv_heads, per_tile = kTileRows / G, units = b.num_seqs + b.num_groups;
    if (tid == 0) { cost = row_cost = 0; totals[0] = totals[1] = totals[2] = 0; }
    __syncthreads();
    unsigned long long mine = 0, mine_rows = 0;
    for (int u = tid; u < units; u += kPlanThreads) {
        const UnitRange r = unit_range(b, c, u);
        mine += (unsigned long long)((r.nt + per_tile - 1) / per_tile) * (unsigned)(r.k1 - r.k0);
        mine_rows += (unsigned long long)r.nt * G * (unsigned)(r.k1 - r.k0);
    }
    atomicAdd(&cost, mine);
    atomicAdd(&row_cost, mine_rows);
    __syncthreads();
    const int target = row_cost / kFewRows <= cost ? kFewItems : kTargetItems;
    const unsigned long long each = cost * (unsigned)b.kv_heads / target + 1;
    const int chunk = each > 0x7fffff00ull ? 0x7fffff00
                                           : max(kMinChunk, (int)((each + kChunkStep - 1) / kChunkStep) * kChunkStep);

    // first item, first row and cost in front of every unit: running sums over blocks of units
    for (int u0 = 0; u0 < units; u0 += kPlanThreads) {
        const int u = u0 + tid;
        long long items = 0, rows = 0, costs = 0;
        PlanUnit pu{};
        if (u < units) {
            const UnitRange r = unit_range(b, c, u);
            pu.tiles = (r.nt + per_tile - 1) / per_tile;
            pu.splits = r.nt > 0 ? (int)(((int64_t)(r.k1 - r.k0) + chunk - 1) / chunk) : 0;
            items = (long long)pu.tiles * pu.splits;
            rows = (long long)r.nt * G * pu.splits;
            pu.cost = min(chunk, r.k1 - r.k0) + kItemCost;
            costs = items * pu.cost;
        }
        long long si = items, sr = rows, sc = costs;
        for (int d = 1; d < 64; d <<= 1) {
            const long long ai = __shfl_up(si, d), ar = __shfl_up(sr, d), ac = __shfl_up(sc, d);
            if ((tid & 63) >= d) { si += ai; sr += ar; sc += ac; }
        }
        if ((tid & 63) == 63) { scan[0][tid >> 6] = si; scan[1][tid >> 6] = sr; scan[2][tid >> 6] = sc; }
        __syncthreads();
        long long bi = totals[0], br = totals[1], bc = totals[2];
        for (int w = 0; w < (tid >> 6); ++w) { bi += scan[0][w]; br += scan[1][w]; bc += scan[2][w]; }
        if (u < units) {
            pu.first_item = (int)(bi + si - items);
            pu.first_row = (int)(br + sr - rows);
            pu.first_cost = bc + sc - costs;
            p.units[u] = pu;
        }
        __syncthreads();
        if (tid == kPlanThreads - 1) { totals[0] = bi + si; totals[1] = br + sr; totals[2] = bc + sc; }
        __syncthreads();
    }
    // (arrays that contradict each other, like starts that fall, can ask for more than there is room for)
    const bool fits = totals[0] * b.kv_heads <= max_items && totals[1] <= max_rows;
    const int n = fits ? (int)totals[0] * b.kv_heads : 0, rows1 = fits ? (int)totals[1] : 0;
    if (tid == 0) {
        PlanHeader &h = *p.head;
        h.magic = kPlanMagic;
        h.num_tokens = b.num_tokens; h.num_seqs = b.num_seqs; h.num_groups = b.num_groups;
        h.heads = b.heads; h.kv_heads = b.kv_heads; h.head_dim = b.head_dim;
        h.max_len = c.max_len; h.table_width = c.table_width; h.page_shift = c.page_shift;
        h.num_items = n; h.rows = rows1;
    }
    // the items at which so many eighths of the cost are reached, of groups and of sequences
    if (tid <= kDies || (tid >= 64 && tid <= 64 + kDies)) {
        const bool own = tid >= 64;
        const int die = tid & 63, u0 = own ? b.num_groups : 0, u1 = own ? units : b.num_groups;
        const int end = u1 == units ? n : min(p.units[u1].first_item * b.kv_heads, n);
        int at = end;
        if (n > 0 && u0 < u1 && die < kDies) {
            const long long c0 = p.units[u0].first_cost, c1 = u1 == units ? totals[2] : p.units[u1].first_cost;
            const long long want = c0 * b.kv_heads + (c1 - c0) * b.kv_heads / kDies * die;
            int lo = u0, hi = u1 - 1;
            while (lo < hi) {
                const int mid = (lo + hi + 1) / 2;
                if (p.units[mid].first_cost * b.kv_heads <= want) lo = mid;
                else hi = mid - 1;
            }
            const PlanUnit pu = p.units[lo];
            at = pu.first_item * b.kv_heads + (pu.cost > 0 ? (int)((want - pu.first_cost * b.kv_heads) / pu.cost) : 0);
        }
        p.head->die_start[own][die] = clampi(at, 0, end);
    }

    for (int i = tid; i < n; i += kPlanThreads) {
        int lo = 0, hi = units - 1;      // the last unit that starts at or before item i (units without items share a start)
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if (p.units[mid].first_item * b.kv_heads <= i) lo = mid;
            else hi = mid - 1;
        }
        const PlanUnit pu = p.units[lo];
        const UnitRange r = unit_range(b, c, lo);
        // tiles that read the same keys are neighbours, then the heads, then the chunks
        const int at = i - pu.first_item * b.kv_heads, tile = at % pu.tiles, head = at / pu.tiles % b.kv_heads, split = at / pu.tiles / b.kv_heads;
        PlanItem it{};
        it.t0 = r.t0 + tile * per_tile;
        it.nt = min(per_tile, r.nt - tile * per_tile);
        it.k0 = r.k0 + (int)min((int64_t)split * chunk, (int64_t)(r.k1 - r.k0));
        it.k1 = (int)min((int64_t)it.k0 + chunk, (int64_t)r.k1);
        it.seq = r.seq;
        it.head = head;
        const bool direct = lo >= b.num_groups && pu.splits == 1 && r.k0 == 0;
        it.base = direct ? -1 : head * rows1 + pu.first_row + (split * r.nt + tile * per_tile) * G;
        p.items[i] = it;
    }

    for (int t = tid; t < b.num_tokens; t += kPlanThreads) {
        PlanToken pt{};
        const int s = b.token_seq[t];
        if (fits && (uint32_t)s < (uint32_t)b.num_seqs) {
            const UnitRange r = unit_range(b, c, b.num_groups + s);
            if (t >= r.t0 && t < r.t0 + r.nt) {
                const PlanUnit pu = p.units[b.num_groups + s];
                pt.limit = clampi(b.token_pos[t], -1, r.k1 - 1) + 1;
                pt.own_splits = pu.splits;
                pt.own_stride = r.nt * G;
                pt.own_base = pu.first_row + (t - r.t0) * G;
                pt.direct = pu.splits == 1 && r.k0 == 0;
                const int g = group_of(b, s);
                if (g >= 0) {
                    const UnitRange q = unit_range(b, c, g);
                    const PlanUnit qu = p.units[g];
                    if (t >= q.t0 && t < q.t0 + q.nt) {
                        pt.pre_splits = qu.splits;
                        pt.pre_stride = q.nt * G;
                        pt.pre_base = qu.first_row + (t - q.t0) * G;
                    }
                }
            }
        }
        p.tokens[t] = pt;
    }
}

// Whether the plan in memory was made for the batch of this call.
__device__ __forceinline__ bool plan_fits(const AttendArgs &a)
{
    const PlanHeader &h = *a.plan.head;
    const BatchArgs &b = a.batch;
    return h.magic == kPlanMagic && h.num_tokens == b.num_tokens && h.num_seqs == b.num_seqs && h.num_groups == b.num_groups &&
           h.heads == b.heads && h.kv_heads == b.kv_heads && h.head_dim == b.head_dim && h.max_len == a.cache.max_len &&
           h.table_width == a.cache.table_width && h.page_shift == a.cache.page_shift;
}

// ---- items ------------------------------------------------------------------------------------

typedef __attribute__((address_space(3))) vec<short, 4> lds_short4;

template <typename T> struct Mfma;
template <> struct Mfma<bf16_t> {
    static __device__ __forceinline__ vec<float, 16> run(vec<bf16_t, 8> a, vec<bf16_t, 8> b, vec<float, 16> c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    }
};
template <> struct Mfma<fp16_t> {
    static __device__ __forceinline__ vec<float, 16> run(vec<fp16_t, 8> a, vec<fp16_t, 8> b, vec<float, 16> c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
    }
};

// Where the 16-byte piece `c` of row `r` of a staged tile is: rows that the lanes of one LDS instruction read lie in
// different banks.  Keys are read a row per lane (32 rows, the same piece), values four rows at a time (four pieces).
template <int CH> __device__ __forceinline__ constexpr int key_turn(int r) { return CH == 8 ? (r >> 1) & 7 : r & 15; }
template <int CH> __device__ __forceinline__ constexpr int value_turn(int r) { return CH == 8 ? ((r >> 1) & 1) << 2 : (r & 3) << 2; }

// The maximum of a row that has seen keys, and no score but minus infinity: less than any other's, so that beside other parts
// it counts for nothing, and alone it is told from a row that has seen no key.
constexpr float kNothing = -3.402823466e38f;

// What the weighted sum is multiplied by.  A row without any key has zeros; one with scores of minus infinity alone has weights
// of 0 by 0, so NaN; NaN stays.
__device__ __forceinline__ float one_by(float m, float l)
{
    return l > 0 ? 1.0f / l : l == 0 && m == -INFINITY ? 0.0f : NAN;
}

// exp2 on the hardware's unit: 1 ulp of 32 bits, and 0 for -infinity.
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// The greater of a lane's value and that of the lane 32 away.  (Swapping the upper half of one copy with the lower half of
// another leaves both values in the two of every lane.)
__device__ __forceinline__ float max_of_halves(float x)
{
    const uint32_t v = __float_as_uint(x);
    const auto y = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
}

// Zeros in the place of infinities and NaN among eight values; whether there were any.
template <typename T> __device__ __forceinline__ bool take_out(vec<uint32_t, 4> &v)
{
    constexpr uint32_t kExponent = std::is_same<T, bf16_t>::value ? 0x7f80 : 0x7c00;
    bool any = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bool lo = (v[i] & kExponent) == kExponent, hi = (v[i] >> 16 & kExponent) == kExponent;
        v[i] &= (lo ? 0 : 0xffffu) | (hi ? 0 : 0xffff0000u);
        any |= lo | hi;
    }
    return any;
}

typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(1))) void global_void;

constexpr float kSlack = 8.0f;       // halvings
// How far below a row's maximum its reference is taken: weights of fp16 have their full bits down to 2^-14, and 131,072 keys
// 25.5 halvings below one were counted in the sum but not in the product, 0.28% of the row.  Up to 2^15 there is room, so that
// border is 2^-21 or less of the greatest weight.
template <typename T> constexpr float kRaise = std::is_same<T, fp16_t>::value ? 7.0f : 0.0f;
constexpr float kFused = 4194304.0f; // 2^22: references beyond it and products that are not rounded do not go together

// s * scale - ref with the product rounded, as a maximum's is.
__device__ __forceinline__ float apart(float s, float scale, float ref)
{
#pragma clang fp contract(off)
    const float t = s * scale;
    return t - ref;
}

// A workgroup of four waves takes items of up to 128 rows, 32 to a wave.  With K the A operand, S^T = K Q^T leaves a lane
// with scores of ONE row (its column), so the running maximum and sum are a lane's own, and P^T is in registers where
// the B operand of O^T = V^T P^T wants it: key slots of the second product are numbered as the first one leaves them.
// V^T's rows come from LDS through the transposing read.  A tile of keys and values is loaded straight into LDS while the
// one before it is computed; where its rows are (the page table's entries) is looked up two tiles ahead, because the
// two trips to memory in a row take longer than a tile.
// What bounds it (bf16, 32 query heads on 8 KV heads of 128 dimensions; both kernels together): memory where few rows see
// many keys, one token behind 131,072 keys 107 us, 5.0 TB/s, 256 tokens behind four prefixes of up to 32,768 and own parts of
// up to 2048 370 to 380 us, 4.7 TB/s (a large copy: 4.9); issue where tiles are full, prompts of up to 512 tokens behind 16,000
// keys (fp16, on 4 KV heads) 830 to 880 us from card to card, 710 to 750 TFLOP/s: 6.5 other vector instructions come to a
// product, the matrix units work 47% of the time and the vector units 50%, so hardly anything of one is hidden behind the
// other.  Few short sequences wait for the chain of loads from the plan to the first tile: four of up to 700 keys 11.1 us, of
// kernels 7.5 and the merge's 4.4.  64 dimensions: 131,072 keys 50 us, prompts 500; 256 (255 + 166 registers, one wave to a
// SIMD): 232 and 2470.
template <typename T, int D>
__global__ __launch_bounds__(256, D == 256 ? 1 : 2) void k_attend_items(AttendArgs a)
{
    constexpr int KB = D == 256 ? 32 : 64, CH = D / 8, LOADS = KB * CH / 256, ROW = D * 2;
    __shared__ uint4 lk0[KB * CH], lv0[KB * CH], lk1[KB * CH], lv1[KB * CH];
    __shared__ int64_t where[4][KB];      // of the next tiles' rows, in pieces (of what is not there: any that is)
    constexpr int MINE = KB / 4;          // rows of a tile that each wave looks up
    typedef std::conditional_t<MINE == 16, uint16_t, uint8_t> Seen;
    __shared__ __align__(8) Seen seen[4][4];      // which of them are there
    __shared__ int reach[4], least[4];
    __shared__ int odd;                   // values were taken out of a tile
    if (!plan_fits(a)) return;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 31, half = lane >> 5;
    const int G = a.batch.heads / a.batch.kv_heads;
    const uint32_t inv_g = 65536 / G + 1;          // r / G for r < 128
    const uint4 *kp = (const uint4 *)a.cache.k, *vp = (const uint4 *)a.cache.v;
    const int page_mask = (1 << a.cache.page_shift) - 1;
    // where a lane reads in a staged tile: pieces of a key by kk, of a value by dt
    const int key_at = col * ROW + ((half ^ key_turn<CH>(col)) << 4);
    const int vrow = half * 4 + (lane & 15) / 4;
    const int value_at = vrow * ROW + (((((lane >> 4) & 1) * 2 + (lane & 3) / 2) ^ value_turn<CH>(vrow)) << 4) + (lane & 1) * 8;

    // Workgroups go to the dies in turn; each die takes a stretch of the groups' items, and behind them one of the
    // sequences', so that neighbouring items (the tiles that read the same keys) meet in one L2 and are there at the same
    // time.  Stretches are of equal cost as the plan counts it.  Of 256 sequences behind 32k prefixes: one stretch of both kinds to a die 458 us
    // (some dies wait for their products, the others for an eighth of the memory's rate each), the kinds in turns 511 (tiles
    // of the same keys drift apart), this 443.  (All three before other changes.)
    const int die = blockIdx.x & (kDies - 1), step = gridDim.x / kDies;
    const int first0 = a.plan.head->die_start[0][die], first1 = a.plan.head->die_start[1][die];
    const int n0 = a.plan.head->die_start[0][die + 1] - first0, n = n0 + a.plan.head->die_start[1][die + 1] - first1;
    for (int i = blockIdx.x / kDies; i < n; i += step) {
        const PlanItem it = a.plan.items[i < n0 ? first0 + i : first1 + i - n0];
        const int rows = it.nt * G;
        const int r = wave * 32 + col;
        const bool valid = r < rows;
        const int rt = (int)((uint32_t)r * inv_g >> 16), token = it.t0 + rt, head = it.head * G + r - rt * G;
        const int lim = valid ? min(a.plan.tokens[token].limit, it.k1) : 0;
        vec<T, 8> q[D / 16];
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
            q[kk] = vec<T, 8>{};
            if (valid) q[kk] = *(const vec<T, 8> *)((const T *)a.q + token * a.q_token_stride + head * a.q_head_stride + kk * 16 + half * 8);
        }
        // How far the wave's rows see: none (hi), all (lo).  Rows that see nothing of the item (padding, sequences that end in
        // front of it) go along with the others and are set to nothing at the end: counted in lo they would make every tile
        // one that rows see differently.
        int hi = lim, lo = lim > it.k0 ? lim : 0x7fffffff;
        for (int d = 1; d < 32; d <<= 1) { hi = max(hi, __shfl_xor(hi, d)); lo = min(lo, __shfl_xor(lo, d)); }
        hi = __builtin_amdgcn_readfirstlane(hi);
        lo = __builtin_amdgcn_readfirstlane(lo);
        __syncthreads();
        if (lane == 0) { reach[wave] = hi; least[wave] = lo; }
        if (tid == 0) odd = 0;
        __syncthreads();
        const int end = max(max(reach[0], reach[1]), max(reach[2], reach[3]));
        const int all = min(min(least[0], least[1]), min(least[2], least[3]));
        const int odd_from = all < end ? all - KB : 0x7fffffff;      // in tiles behind this key rows differ in what they see

        vec<float, 16> o[D / 32];
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) o[dt] = vec<float, 16>{};
        float m = -INFINITY, l = 0;           // reference and sum
        bool far = false;                     // a reference of the wave's is beyond kFused
        int first_there = 0x7fffffff;         // the first key that is there

        const int32_t *table = a.cache.table + (int64_t)it.seq * a.cache.table_width;
        auto entry = [&](int kt) {
            const int key = kt + wave * MINE + lane;
            const int page = table[min(key, end - 1) >> a.cache.page_shift];      // (no branch: it would wait for the load)
            return key < end ? page : -1;
        };
        auto note = [&](int kt, int64_t page, int slot) {
            const int key = kt + wave * MINE + lane;
            const bool there = lane < MINE && page >= 0 && page < a.cache.num_pages;
            if (lane < MINE)
                where[slot][wave * MINE + lane] = there
                    ? (page * a.cache.page_stride + (int64_t)(key & page_mask) * a.cache.slot_stride + it.head * a.cache.head_stride) / 8 : 0;
            const unsigned long long bits = __ballot(there);
            if (lane == 0) seen[slot][wave] = (Seen)bits;
        };
        auto load = [&](auto buf, int slot) {
            uint4 *const lk = buf.value ? lk1 : lk0, *const lv = buf.value ? lv1 : lv0;
#pragma unroll
            for (int x = 0; x < LOADS; ++x) {
                const int row = (x * 256 + wave * 64 + lane) / CH, c = lane % CH;
                const int64_t at = where[slot][row];
                __builtin_amdgcn_global_load_lds((global_void *)(kp + at + (c ^ key_turn<CH>(row))), (lds_void *)(lk + x * 256 + wave * 64), 16, 0, 0);
                __builtin_amdgcn_global_load_lds((global_void *)(vp + at + (c ^ value_turn<CH>(row))), (lds_void *)(lv + x * 256 + wave * 64), 16, 0, 0);
            }
        };
        auto compute = [&](auto buf, int kt, int slot) {
            const char *const lk = (const char *)(buf.value ? lk1 : lk0);
            char *const lv = (char *)(buf.value ? lv1 : lv0);
            unsigned long long bits = ~0ull;
            __builtin_memcpy(&bits, seen[slot], sizeof(seen[slot]));
            bits = (unsigned long long)__builtin_amdgcn_readfirstlane((int)(bits >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)bits);
            const unsigned long long any = KB == 64 ? bits : (uint32_t)bits;
            if (any && first_there == 0x7fffffff) first_there = kt + __builtin_ctzll(any);
            // Values that nothing sees may be no numbers: zeros.  Where some rows see keys that others do not, values that
            // are no numbers are taken out, too, and added at the end where they are seen (a weight of zero would make
            // NaN of them).
            const bool some = kt > odd_from;
            if (bits != ~0ull || some) {
                for (int x = tid; x < KB * CH; x += 256) {
                    vec<uint32_t, 4> v = ((const vec<uint32_t, 4> *)lv)[x];
                    if (bits >> (x / CH) & 1) {
                        if (!some || !take_out<T>(v)) continue;
                        odd = 1;
                    } else {
                        v = vec<uint32_t, 4>{};
                    }
                    ((vec<uint32_t, 4> *)lv)[x] = v;
                }
                __syncthreads();
            }
            if (kt >= hi) return;
            // All scores of the tile, so that the rows' maxima are looked at once, then the weights and the product with the
            // values thirty-two keys at a time.  The order within is the compiler's: with operands read a phase ahead and the
            // phases held apart, prompts behind 16k keys 895 us, so 853; one sequence of 131k keys 115, so 107.
            int key_from = key_at, value_from = value_at;
            asm volatile("" : "+v"(key_from), "+v"(value_from));      // (a dozen exclusive-ors a tile instead of as many registers)
            constexpr int NB = KB / 32;
            vec<float, 16> s[NB];
#pragma unroll
            for (int kb = 0; kb < NB; ++kb) {
                s[kb] = vec<float, 16>{};
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk)
                    s[kb] = Mfma<T>::run(*(const vec<T, 8> *)(lk + (key_from ^ (kk << 5)) + kb * 32 * ROW), q[kk], s[kb]);
            }
            if (kt + KB > lo || bits != ~0ull) {
#pragma unroll
                for (int kb = 0; kb < NB; ++kb) {
                    const int left = lim - kt - kb * 32 - 4 * half;          // (rows counted from the lane's first)
                    const uint32_t b = (uint32_t)(bits >> (kb * 32 + 4 * half));
#pragma unroll
                    for (int x = 0; x < 16; ++x) {
                        const int row = 8 * (x / 4) + x % 4;
                        const bool vis = row < left && (b & 1u << row);
                        s[kb][x] = vis ? s[kb][x] : -INFINITY;
                    }
                }
            }
            float top = s[0][0];
#pragma unroll
            for (int x = 1; x < 16 * NB; ++x) top = fmaxf(top, s[x / 16][x % 16]);
            top = max_of_halves(top);
            // The reference of the weights follows the maximum only when that is kSlack further above it than it was: weights
            // up to 2^(kSlack + kRaise) lose nothing in either type, and the results are scaled once or twice a row, not
            // whenever one of a wave's rows has a new maximum (in two tiles of five over 8000 keys).
            float scale = a.scale_log2;
            float ref = m == -INFINITY ? 0.0f : m;      // (a row that has seen nothing yet)
            if (__any(apart(top, scale, m) > kSlack + kRaise<T>) || far) {      // (not against a sum, which is rounded)
                const float m2 = fmaxf(m, apart(top, scale, kRaise<T>));
                const float f = m2 == -INFINITY ? 1.0f : exp2_fast(m - m2);
                m = m2;
                l *= f;
#pragma unroll
                for (int dt = 0; dt < D / 32; ++dt) o[dt] *= f;
                ref = m == -INFINITY ? 0.0f : m;
                // Weights are exp2 of one fused operation a score, and the reference is a product that was rounded: by less
                // than an eighth up to 2^22, by 8 and more from 2^27 on, where a row's weights would all be infinite or 0.
                far = __any(fabsf(m) > kFused && m > -INFINITY);
                if (far) {
#pragma unroll
                    for (int x = 0; x < 16 * NB; ++x) s[x / 16][x % 16] = apart(s[x / 16][x % 16], scale, ref);
                    scale = 1.0f;
                    ref = 0.0f;
                }
            }
#pragma unroll
            for (int kb = 0; kb < NB; ++kb) {
                union { vec<short, 4> h[2]; vec<T, 8> v; } vf[D / 32][2];
#pragma unroll
                for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        const char *at = lv + (value_from ^ (dt << 6)) + (kb * 2 + g) * 16 * ROW;
                        vf[dt][g].h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4 *)at);
                        vf[dt][g].h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4 *)(at + 8 * ROW));
                    }
                vec<T, 8> pt[2];
#pragma unroll
                for (int x = 0; x < 16; x += 2) {
                    const vec<float, 2> e = {exp2_fast(s[kb][x] * scale - ref), exp2_fast(s[kb][x + 1] * scale - ref)};
                    l += e[0];
                    l += e[1];
                    // Rounded to 16 bits, half a step each, because the matrix instruction takes both sides in one type; the sum
                    // takes them before.  Against 64 bits results are then off by 2.3e-3 of their norm in bf16 and 2.9e-4
                    // in fp16, where weights of 32 bits give 1.7e-3 and 2.1e-4 (the rounding of the result alone).  What is
                    // left of each weight in a second product would double the products with the values.
                    const vec<T, 2> y = __builtin_convertvector(e, vec<T, 2>);
                    pt[x / 8][x % 8] = y[0];
                    pt[x / 8][x % 8 + 1] = y[1];
                }
#pragma unroll
                for (int g = 0; g < 2; ++g)
#pragma unroll
                    for (int dt = 0; dt < D / 32; ++dt) o[dt] = Mfma<T>::run(vf[dt][g].v, pt[g], o[dt]);
            }
        };
        if (end > it.k0) {
            note(it.k0, entry(it.k0), 0);
            note(it.k0 + KB, entry(it.k0 + KB), 1);
            __syncthreads();
            load(std::integral_constant<int, 0>(), 0);
        }
        for (int kt = it.k0, t = 0; kt < end; kt += KB, ++t) {
            auto tile = [&](auto buf) {
                __builtin_amdgcn_s_waitcnt(0x0f70);       // this tile is there
                __syncthreads();
                const int e = entry(kt + 2 * KB);
                load(std::integral_constant<int, 1 - buf.value>(), (t + 1) & 3);      // (behind the last tile: any row)
                compute(buf, kt, t & 3);
                note(kt + 2 * KB, e, (t + 2) & 3);
            };
            tile(std::integral_constant<int, 0>());
            kt += KB;
            ++t;
            if (kt >= end) break;
            tile(std::integral_constant<int, 1>());
        }
        __builtin_amdgcn_s_waitcnt(0x0f70);       // (nothing is under way to LDS when the next item or the end comes)

        __syncthreads();
        if (odd) {      // the values that were taken out, of the tiles that they were taken out of
            for (int key = it.k0 + max(0, odd_from + KB - it.k0) / KB * KB; key < lim; ++key) {
                const int64_t page = table[key >> a.cache.page_shift];
                if (page < 0 || page >= a.cache.num_pages) continue;
                const T *v = (const T *)a.cache.v + page * a.cache.page_stride + (key & page_mask) * a.cache.slot_stride +
                             it.head * a.cache.head_stride + 4 * half;
#pragma unroll
                for (int x = 0; x < D / 8; ++x) {
                    const vec<T, 4> y = *(const vec<T, 4> *)(v + 8 * x);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (!(fabsf((float)y[e]) < INFINITY)) o[x / 4][x % 4 * 4 + e] += (float)y[e];
                }
            }
        }
        l += __shfl_xor(l, 32);
        int limit = lim;      // (compared again: the answer kept through the tiles takes prompts from 837 us to 870)
        asm volatile("" : "+v"(limit));
        if (limit <= it.k0) {
            m = -INFINITY;
            l = 0;
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt) o[dt] = vec<float, 16>{};
        }
        // A sum of 0 is that of a row that sees no key, or of one whose scores are all minus infinity.
        if (l == 0 && lim > first_there) m = kNothing;
        if (valid && it.base < 0) {
            const float f = one_by(m, l);
            T *out = (T *)a.out + token * a.out_token_stride + head * a.out_head_stride;
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    vec<T, 4> y;
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[e] = (T)(o[dt][4 * x + e] * f);
                    *(vec<T, 4> *)(out + dt * 32 + 8 * x + 4 * half) = y;
                }
        } else if (valid) {
            const int64_t row = (int64_t)it.base + r;
            if (half == 0) a.part_ml[row] = float2{m, l};
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    *(vec<float, 4> *)(a.part_o + row * D + dt * 32 + 8 * x + 4 * half) =
                        vec<float, 4>{o[dt][4 * x], o[dt][4 * x + 1], o[dt][4 * x + 2], o[dt][4 * x + 3]};
        }
    }
}

// ---- merge ------------------------------------------------------------------------------------

// D/4 threads side by side take four dimensions of a (token, query head) each.  A workgroup takes ROWS of those; the
// threads that are left over take further splits, merged through LDS at the end.  Bound by the reads of the results, from
// L2 and memory: 80,000 rows of three splits 25 us.  One row to a workgroup for few rows
// (which may have a hundred splits each), as many as fit for many: those 80,000 rows took 145 us with one row each.
template <typename T, int D, int ROWS>
__global__ __launch_bounds__(256) void k_attend_merge(AttendArgs a, int64_t first_item)
{
    constexpr int W = D / 4, LANES = 256 / W / ROWS;
    __shared__ float lm[ROWS][LANES], ll[ROWS][LANES];
    __shared__ vec<float, 4> lo[LANES > 1 ? ROWS * LANES : 1][W];
    const int sub = threadIdx.x / (W * LANES), d = threadIdx.x % W, lane = threadIdx.x / W % LANES;
    const int64_t item = first_item + (int64_t)blockIdx.x * ROWS + sub;
    const bool there = item < (int64_t)a.batch.num_tokens * a.batch.heads;
    const int token = there ? (int)(item / a.batch.heads) : 0, head = there ? (int)(item % a.batch.heads) : 0;
    T *out = (T *)a.out + token * a.out_token_stride + head * a.out_head_stride + d * 4;
    if (!plan_fits(a)) {
        if (there && lane == 0) *(vec<T, 4> *)out = vec<T, 4>{(T)NAN, (T)NAN, (T)NAN, (T)NAN};
        return;
    }
    const PlanToken pt = a.plan.tokens[token];
    const int G = a.batch.heads / a.batch.kv_heads;
    const int64_t first = (int64_t)(head / G) * a.plan.head->rows + head % G;
    const bool work = there && !pt.direct;
    float m = -INFINITY, l = 0;
    vec<float, 4> o = vec<float, 4>{};
    auto join = [&](float m1, float l1, vec<float, 4> o1) {
        if (m1 == -INFINITY && l1 == 0) return;        // nothing seen
        if (m == -INFINITY && l == 0) {                // nothing so far
            m = m1; l = l1; o = o1;
            return;
        }
        // (a sum of NaN with a maximum of -infinity, of scores that are all NaN, stays NaN times 0)
        const float m2 = fmaxf(m, m1), f = exp2_fast(m - m2), g = exp2_fast(m1 - m2);
        o = o * f + o1 * g;
        l = l * f + l1 * g;
        m = m2;
    };
    if (work) {
        const int splits = pt.own_splits + pt.pre_splits;
        auto row_of = [&](int s) {
            return first + (s < pt.pre_splits ? pt.pre_base + (int64_t)s * pt.pre_stride
                                              : pt.own_base + (int64_t)(s - pt.pre_splits) * pt.own_stride);
        };
        constexpr int AHEAD = 4;      // splits under way at a time
        for (int s0 = lane; s0 < splits; s0 += AHEAD * LANES) {
            float2 ml[AHEAD];
            vec<float, 4> x[AHEAD];
#pragma unroll
            for (int e = 0; e < AHEAD; ++e) {
                const int s = s0 + e * LANES;
                const int64_t row = row_of(s < splits ? s : s0);
                ml[e] = s < splits ? a.part_ml[row] : float2{-INFINITY, 0};
                x[e] = *(const vec<float, 4> *)(a.part_o + row * D + d * 4);
            }
#pragma unroll
            for (int e = 0; e < AHEAD; ++e) join(ml[e].x, ml[e].y, x[e]);
        }
    }
    if (LANES > 1) {
        if (d == 0) { lm[sub][lane] = m; ll[sub][lane] = l; }
        lo[sub * LANES + lane][d] = o;
        __syncthreads();
        if (lane != 0) return;
        for (int s = 1; s < LANES; ++s) join(lm[sub][s], ll[sub][s], lo[sub * LANES + s][d]);
    }
    const float f = one_by(m, l);
    if (work) *(vec<T, 4> *)out = vec<T, 4>{(T)(o[0] * f), (T)(o[1] * f), (T)(o[2] * f), (T)(o[3] * f)};
}

template <typename T, int D>
hipError_t attend(const AttendArgs &a, int64_t max_items, hipStream_t s)
{
    // (twice the items, because dies with shorter ones have more of them)
    const int grid = ((int)(max_items < 1024 ? 2 * max_items : 2048) / kDies + 1) * kDies;
    k_attend_items<T, D><<<grid, 256, 0, s>>>(a);
    if (hipError_t e = hipGetLastError()) return e;
    const int64_t rows = (int64_t)a.batch.num_tokens * a.batch.heads;
    constexpr int MANY = 256 / (D / 4);
    if (rows < 32768) {
        k_attend_merge<T, D, 1><<<(unsigned)rows, 256, 0, s>>>(a, 0);
        return hipGetLastError();
    }
    for (int64_t first = 0; first < rows; first += kMostGroups * MANY) {
        const dim3 grid((unsigned)std::min(kMostGroups, (rows - first + MANY - 1) / MANY));
        k_attend_merge<T, D, MANY><<<grid, 256, 0, s>>>(a, first);
        if (hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}

template <typename T>
hipError_t attend(const AttendArgs &a, int64_t max_items, hipStream_t s)
{
    switch (a.batch.head_dim) {
    case 64: return attend<T, 64>(a, max_items, s);
    case 128: return attend<T, 128>(a, max_items, s);
    default: return attend<T, 256>(a, max_items, s);
    }
}

}  // namespace

hipError_t launch_plan(const BatchArgs &b, const CacheArgs &c, const PlanView &p, const PlanSizes &z, hipStream_t s)
{
    k_plan<<<1, kPlanThreads, 0, s>>>(b, c, p, (int)z.max_items, (int)z.max_rows);
    return hipGetLastError();
}

hipError_t launch_attend(const AttendArgs &a, int32_t type, int64_t max_items, hipStream_t s)
{
    return type == INFAAS_SEL_TYPE_BF16 ? attend<bf16_t>(a, max_items, s) : attend<fp16_t>(a, max_items, s);
}

}  // namespace infaas
