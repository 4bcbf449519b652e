// Drawing a token of every row of logits (infaas_sel_exec_sample).
#include "exec.h"

namespace infaas {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kMostSegments = 4352;          // of a row: 2^20 logits of 32 bits at any alignment are 4112
constexpr int kMostListed = 2048;            // candidates that are put in order in LDS, two to a thread
constexpr int kBuckets = 2048;               // of logits by their distance from the greatest
constexpr int kShift = 43;                   // a weight of 1 is 2^43: 2^20 of them stay below 2^63
constexpr float kFar = 44.0f;                // in halvings: weights further down are 0 units
constexpr uint32_t kNever = 0x007fffffu;     // order key of -infinity
constexpr int kLastIndex = 0x7fffffff;
constexpr unsigned long long kRaw = 0x4330000000000000ull;   // the bits of 2^52

typedef unsigned long long u64;

// Logits that are numbers as 32-bit keys in their order: equal logits (-0 and +0, too) have equal keys.
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t k) { return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k); }

// Weights exp((x - top) / temperature) in units of 2^-43: 2^t, t = (x - top) * log2(e) / temperature, as 2^round(t) times
// the Taylor series of 2^f = e^(f ln 2), |f| <= 1/2, to the eleventh power: what is left out is 0.347^12 / 12! = 6e-15 of
// it, less than the rounding to units.  Among +infinities 1.
struct Weights {
    double top, halvings;
    bool infinite;
    // The units plus kRaw (for sums of many: one subtraction at the end instead of one each).  A weight is rounded to units
    // by adding 2^52 to the double, whose bits are then those of the units behind the exponent; t below the range gives 0.
    __device__ __forceinline__ u64 raw(float x) const
    {
        if (infinite) return kRaw + (x == INFINITY ? 1ull << kShift : 0);
        const double t = ((double)x - top) * halvings;
        constexpr double whole = 6755399441055744.0 + kShift;      // 1.5 * 2^52: adding it rounds to an integer, in the low bits
        const double r = t + whole, f = t - (r - whole);
        constexpr double c[] = {1.0, 0.69314718055994531, 0.24022650695910072, 0.055504108664821580, 0.0096181291076284772,
                                0.0013333558146428443, 1.5403530393381610e-4, 1.5252733804059840e-5, 1.3215486790144309e-6,
                                1.0178086009239699e-7, 7.0549116208011233e-9, 4.4455382718708116e-10};
        double p = c[11];
#pragma unroll
        for (int i = 10; i >= 0; --i) p = __builtin_fma(p, f, c[i]);
        const u64 scaled = __double_as_longlong(p) + ((u64)(uint32_t)__double_as_longlong(r) << 52);
        const u64 bits = __double_as_longlong(__longlong_as_double(scaled) + 4503599627370496.0);
        return t > -(double)kFar ? bits : kRaw;
    }
    __device__ __forceinline__ u64 operator()(float x) const { return raw(x) - kRaw; }
};

// What is kept: everything above `value`, and of the tokens at it those numbered up to `last`.  (Never NaN.)
struct Kept {
    float value;
    int last;
    __device__ __forceinline__ bool has(float x, int i) const { return x > value || (x == value && i <= last); }
};

struct Shared {
    u64 seg[kMostSegments];
    u64 list[kMostListed];
    u64 mass[kBuckets];
    uint32_t count[256];
    u64 wave_sum[kWaves];
    uint32_t wave_count[2][kWaves];
    float wave_top[kWaves];
    uint32_t listed;
    int index;
    u64 left;
};

__device__ __forceinline__ u64 wave_sum(u64 v)
{
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// A row in pieces of 16 bytes, at the addresses that are multiples of 16, a piece per thread at a time, so that the
// pieces of a wave in one round are a segment of the row, and the segments in the order of rounds and waves are in the
// order of tokens. 
template <typename T>
struct Row {
    static constexpr int E = 16 / sizeof(T);
    const T *row;
    int V, shift, rounds;

    __device__ __forceinline__ void init(const T *p, int n)
    {
        row = p;
        V = n;
        shift = (int)((uintptr_t)p / sizeof(T) % E);
        rounds = ((V + shift + E - 1) / E + kThreads - 1) / kThreads;
    }
    __device__ __forceinline__ int first(int piece) const { return piece * E - shift; }
    __device__ __forceinline__ int segments() const { return rounds * kWaves; }
    __device__ __forceinline__ int segment_of(int i) const { return (i + shift) / (E * 64); }

    __device__ __forceinline__ uint4 read(int piece) const
    {
        const int i = first(piece);
        uint4 v;
        if (i >= 0 && i + E <= V) v = *(const uint4 *)(row + i);
        else {
            T x[E];
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = i + e >= 0 && i + e < V ? row[i + e] : (T)-INFINITY;
            __builtin_memcpy(&v, x, 16);
        }
        return v;
    }
    // f(logit, token) of every token of a piece; what is no token counts as -infinity, what is no number may come as it is
    template <typename F> __device__ __forceinline__ void each(uint4 v, int piece, F f) const
    {
        T x[E];
        __builtin_memcpy(x, &v, 16);
#pragma unroll
        for (int e = 0; e < E; ++e) f((float)x[e], first(piece) + e);
    }
    // body(piece's contents, piece, round) for all rounds: those that lie within the row without a look at its ends, the
    // next AHEAD pieces under way while these are worked on; then the one or two others.
    template <typename F> __device__ __forceinline__ void all(F body) const
    {
        constexpr int AHEAD = 16 / E;
        const int lo = shift ? 1 : 0, hi = max(lo, (V + shift) / (E * kThreads)), tid = threadIdx.x;
        if (lo < hi) {
            const T *const from = row - shift;
            uint4 next[AHEAD];
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) next[a] = *(const uint4 *)(from + (int64_t)(min(lo + a, hi - 1) * kThreads + tid) * E);
            for (int r0 = lo; r0 < hi; r0 += AHEAD) {
                uint4 v[AHEAD];
#pragma unroll
                for (int a = 0; a < AHEAD; ++a) v[a] = next[a];
#pragma unroll
                for (int a = 0; a < AHEAD; ++a) next[a] = *(const uint4 *)(from + (int64_t)(min(r0 + AHEAD + a, hi - 1) * kThreads + tid) * E);
#pragma unroll
                for (int a = 0; a < AHEAD; ++a)
                    if (r0 + a < hi) body(v[a], (r0 + a) * kThreads + tid, r0 + a);
            }
        }
#pragma unroll 1
        for (int r = lo ? 0 : hi; r < rounds; r = r < lo ? hi : r + 1) body(read(r * kThreads + tid), r * kThreads + tid, r);
    }
};

// Running sums over v[0 .. n-1] in place (each entry: what is in front of it); returns the total.  All threads.
__device__ u64 scan(Shared &sh, u64 *v, int n)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, each = (n + kThreads - 1) / kThreads;
    u64 sum = 0;
    for (int i = tid * each; i < min(n, (tid + 1) * each); ++i) sum += v[i];
    u64 inc = sum;
    for (int d = 1; d < 64; d <<= 1) {
        const u64 o = __shfl_up(inc, d);
        if (lane >= d) inc += o;
    }
    if (lane == 63) sh.wave_sum[wave] = inc;
    __syncthreads();
    u64 before = inc - sum, all = 0;
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) before += sh.wave_sum[w];
        all += sh.wave_sum[w];
    }
    for (int i = tid * each; i < min(n, (tid + 1) * each); ++i) {
        const u64 x = v[i];
        v[i] = before;
        before += x;
    }
    __syncthreads();
    return all;
}

// Sums of f(logit, token) over the segments, into sh.seg.
template <typename R, typename F> __device__ __forceinline__ void segment_sums(Shared &sh, R &row, F f)
{
    const int wave = threadIdx.x >> 6;
    row.all([&](uint4 v, int piece, int round) {
        u64 c = 0;
        row.each(v, piece, [&](float x, int i) { c += f(x, i); });
        c = wave_sum(c);
        if ((threadIdx.x & 63) == 0) sh.seg[round * kWaves + wave] = c;
    });
    __syncthreads();
}

// The same of all weights from `least` units on.
template <typename R> __device__ __forceinline__ void segment_weights(Shared &sh, R &row, const Weights &wt, u64 least)
{
    const int wave = threadIdx.x >> 6;
    row.all([&](uint4 v, int piece, int round) {
        u64 c = 0;
        if (least <= 1) {
            row.each(v, piece, [&](float x, int) { c += wt.raw(x); });
            c -= R::E * kRaw;
        } else {
            row.each(v, piece, [&](float x, int) {
                const u64 w = wt(x);
                c += w >= least ? w : 0;
            });
        }
        c = wave_sum(c);
        if ((threadIdx.x & 63) == 0) sh.seg[round * kWaves + wave] = c;
    });
    __syncthreads();
}

// The token whose measure f(logit, token), added to those of the tokens with lower numbers, first exceeds `at` (which is
// less than the sum of all).  sh.seg holds the running sums of the segments.  All threads get the answer.
template <typename R, typename F> __device__ int find_in_order(Shared &sh, R &row, u64 at, F f)
{
    const int tid = threadIdx.x, lane = tid & 63, segs = row.segments();
    for (int i = tid; i < segs; i += kThreads) {
        const u64 next = i + 1 < segs ? sh.seg[i + 1] : ~0ull;
        if (sh.seg[i] <= at && at < next) sh.index = i;      // (of segments that add nothing the last: one thread)
    }
    __syncthreads();
    const int seg = sh.index;
    __syncthreads();
    if (tid < 64) {
        const int piece = seg * 64 + lane;
        const uint4 v = row.read(piece);
        u64 mine = 0;
        row.each(v, piece, [&](float x, int i) { mine += f(x, i); });
        u64 inc = mine;
        for (int d = 1; d < 64; d <<= 1) {
            const u64 o = __shfl_up(inc, d);
            if (lane >= d) inc += o;
        }
        u64 before = sh.seg[seg] + inc - mine;
        int found = kLastIndex;
        row.each(v, piece, [&](float x, int i) {
            const u64 w = f(x, i);
            before += w;
            if (w > 0 && before > at) found = min(found, i);
        });
        for (int d = 32; d; d >>= 1) found = min(found, __shfl_xor(found, d));
        if (lane == 0) sh.index = found;
    }
    __syncthreads();
    return sh.index;
}

// Adds (logit, token) to sh.list where `take` is set; counts on beyond the list's end.
__device__ __forceinline__ void put(Shared &sh, bool take, float x, int i)
{
    const u64 mask = __ballot(take);
    if (!mask) return;
    uint32_t base = 0;
    const int lane = threadIdx.x & 63, leader = __ffsll(mask) - 1;
    if (lane == leader) base = atomicAdd(&sh.listed, (uint32_t)__popcll(mask));
    base = __shfl(base, leader) + __popcll(mask & ((1ull << lane) - 1));
    if (take && base < kMostListed) sh.list[base] = (u64)~key_of(x) << 32 | (uint32_t)i;
}

// Puts the n entries of sh.list in order, the greatest logit first, equal ones by number.
__device__ void sort_list(Shared &sh, int n)
{
    int m = 64;
    while (m < n) m *= 2;
    for (int i = n + threadIdx.x; i < m; i += kThreads) sh.list[i] = ~0ull;
    __syncthreads();
    for (int size = 2; size <= m; size *= 2)
        for (int step = size / 2; step; step /= 2) {
            const int t = threadIdx.x;
            if (t < m / 2) {
                const int i = (t / step) * step * 2 + t % step, j = i + step;
                const bool up = (i & size) == 0;
                const u64 x = sh.list[i], y = sh.list[j];
                if ((x > y) == up) { sh.list[i] = y; sh.list[j] = x; }
            }
            __syncthreads();
        }
}
__device__ __forceinline__ float listed(u64 x) { return value_of(~(uint32_t)(x >> 32)); }

// Of the tokens in `within`, from the greatest: the one at which the number of tokens (by_mass: the sum of their
// weights) reaches `target` >= 1, as the border of what is then kept.  If it is never reached, everything is.  Eight bits
// of the key at a time: right for every row, and slow (each of the four passes ends in atomics on few counters), it
// is there for what the lists are too short for.
template <bool by_mass, typename R>
__device__ __forceinline__ Kept select(Shared &sh, R &row, const Weights &wt, Kept within, u64 target)
{
    const int tid = threadIdx.x;
    uint32_t prefix = 0;
    u64 left = target, ties = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = tid; i < 256; i += kThreads) sh.count[i] = 0, sh.mass[i] = 0;
        __syncthreads();
        const uint32_t mask = shift == 24 ? 0u : ~0u << (shift + 8);
        row.all([&](uint4 v, int piece, int) {
            row.each(v, piece, [&](float x, int i) {
                const uint32_t k = key_of(x);
                if ((k & mask) == prefix && x > -INFINITY && within.has(x, i)) {
                    atomicAdd(&sh.count[k >> shift & 255], 1u);
                    if (by_mass) atomicAdd(&sh.mass[k >> shift & 255], wt(x));
                }
            });
        });
        __syncthreads();
        if (tid == 0) {
            int b = 255;
            u64 l = left;
            for (; b >= 0; --b) {
                const u64 here = by_mass ? sh.mass[b] : sh.count[b];
                if (here >= l) break;
                l -= here;
            }
            sh.index = b;
            sh.left = l;
        }
        __syncthreads();
        const int b = sh.index;
        if (b < 0) return within;
        left = sh.left;
        ties = sh.count[b];
        prefix |= (uint32_t)b << shift;
        __syncthreads();
    }
    // of the tokens with this logit the first so many
    const float value = value_of(prefix);
    const u64 m = by_mass ? (left + wt(value) - 1) / wt(value) : left;
    if (m >= ties) return Kept{value, value == within.value ? within.last : kLastIndex};
    auto is = [&](float x, int) -> u64 { return x == value; };
    segment_sums(sh, row, is);
    scan(sh, sh.seg, row.segments());
    return Kept{value, find_in_order(sh, row, m - 1, is)};
}

// A workgroup per row: the greatest logit, then what is kept, by whichever way is short for the row's limits, with the
// sums of its weights by segments, then the segment that the draw falls into.
//   top-k up to kThreads: the k-th of the threads' greatest logits is a bound that k tokens at least reach, and few more;
//     those are listed, put in order, and cut by all limits there.
//   top-p alone: weights summed into buckets of logits; the bucket that the border is in is listed and put in order.
//   neither: nothing to find.
// Where the lists are too short (top-k above kThreads, thousands of equal logits at a border) the border is found eight
// bits at a time.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_sample(SampleArgs a)
{
    __shared__ Shared sh;
    const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, V = a.vocab;
    Row<T> row;
    row.init((const T *)a.logits + r * a.row_stride, V);
    const int segs = row.segments();
    const float t = a.temperature ? a.temperature[r] : 1.0f;
    const float top_p = a.top_p ? a.top_p[r] : 1.0f, min_p = a.min_p && a.min_p[r] > 0 ? a.min_p[r] : 0.0f;
    const bool greedy = !(t > 0) || min_p > 1.0f;
    const int k = a.top_k ? a.top_k[r] : 0;

    if (tid == 0) { sh.listed = 0; sh.index = kLastIndex; }
    float mine = -INFINITY;
    int at_token = kLastIndex;
    if (greedy) row.all([&](uint4 v, int piece, int) { row.each(v, piece, [&](float x, int i) { if (x > mine) { mine = x; at_token = i; } }); });
    else row.all([&](uint4 v, int piece, int) { row.each(v, piece, [&](float x, int) { mine = fmaxf(mine, x); }); });
    float top = mine;
    for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    if (lane == 0) sh.wave_top[wave] = top;
    __syncthreads();
    top = sh.wave_top[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) top = fmaxf(top, sh.wave_top[w]);
    if (top == -INFINITY || greedy) {
        if (mine == top && greedy) atomicMin(&sh.index, at_token);
        __syncthreads();
        if (tid == 0) {
            a.token[r] = top == -INFINITY ? -1 : sh.index;
            if (a.prob) a.prob[r] = top == -INFINITY ? 0.0f : 1.0f;
        }
        return;
    }
    Weights wt;
    wt.top = top;
    wt.infinite = top == INFINITY;
    wt.halvings = 1.4426950408889634 / (double)t;
    // the least weight that is kept, in units: w >= min_p as numbers is rint(2^43 w) >= this but for what is nearer to the
    // border than half a unit
    const u64 least = max((u64)rint((double)min_p * (double)(1ull << kShift)), 1ull);
    const double need_share = (double)top_p;
    auto needed = [&](u64 total) {       // units in front of which a token is still kept
        const double need = ceil(need_share * (double)total);
        return need >= 1.0 ? (u64)need : 1ull;
    };

    Kept kept{-INFINITY, -1};
    bool summed = false;                 // sh.seg holds the sums of what is kept
    auto measure = [&](float x, int i) -> u64 {
        if (!kept.has(x, i)) return 0;
        const u64 w = wt(x);
        return w >= least ? w : 0;
    };
    const bool by_p = top_p < 1.0f, everything = !by_p && !(k > 0 && k < V);
    if (k > 0 && k < V) {
        if (k <= kThreads) {
            uint32_t bound = 0;
            const uint32_t mine_key = key_of(mine);             // the k-th greatest of the threads' greatest, bit by bit
            for (int bit = 31; bit >= (sizeof(T) == 2 ? 13 : 0); --bit) {
                const uint32_t with = bound | 1u << bit;
                const uint32_t c = __popcll(__ballot(mine_key >= with));
                if (lane == 0) sh.wave_count[bit & 1][wave] = c;
                __syncthreads();
                uint32_t all = 0;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) all += sh.wave_count[bit & 1][w];
                if (all >= (uint32_t)k) bound = with;
            }
            // (a bound of no number: fewer threads than k have logits at all)
            const float from = bound <= kNever ? -INFINITY : value_of(bound);
            row.all([&](uint4 v, int piece, int) {
                row.each(v, piece, [&](float x, int i) { put(sh, x >= from && x > -INFINITY, x, i); });
            });
            __syncthreads();
        }
        const int n = (int)sh.listed;
        if (k <= kThreads && n <= kMostListed && n > 0) {
            for (int s = tid; s < segs; s += kThreads) sh.seg[s] = 0;
            sort_list(sh, n);
            if (tid == 0) sh.index = 0;
            u64 *w = sh.mass;            // (as many entries as the list)
            for (int i = tid; i < n; i += kThreads) w[i] = i < k ? wt(listed(sh.list[i])) : 0;
            __syncthreads();
            const u64 total = scan(sh, w, n);
            const u64 need = by_p ? needed(total) : ~0ull;
            for (int i = tid; i < n; i += kThreads) {
                const u64 x = (i + 1 < n ? w[i + 1] : total) - w[i];
                if (i < k && w[i] < need && x >= least) {
                    atomicMax(&sh.index, i);
                    atomicAdd(&sh.seg[row.segment_of((int)sh.list[i])], x);
                }
            }
            __syncthreads();
            const u64 last = sh.list[sh.index];
            kept = Kept{listed(last), (int)last};
            summed = true;
            __syncthreads();
        } else {
            __syncthreads();
            kept = select<false>(sh, row, wt, kept, (u64)k);
            if (by_p) {
                segment_sums(sh, row, [&](float x, int i) -> u64 { return kept.has(x, i) ? wt(x) : 0; });
                kept = select<true>(sh, row, wt, kept, needed(scan(sh, sh.seg, segs)));
            }
        }
    } else if (by_p) {
        const float per = fminf((float)(wt.halvings * (kBuckets / (double)kFar)), 3e38f);
        auto bucket = [&](float x) { return (int)fminf((top - x) * per, (float)(kBuckets - 1)); };
        for (int i = tid; i < kBuckets; i += kThreads) sh.mass[i] = 0;
        __syncthreads();
        if (!wt.infinite)
            row.all([&](uint4 v, int piece, int) {
                row.each(v, piece, [&](float x, int) {
                    const u64 w = wt(x);
                    if (w) atomicAdd(&sh.mass[bucket(x)], w);
                });
            });
        __syncthreads();
        const u64 total = scan(sh, sh.mass, kBuckets);
        const u64 need = needed(total);
        if (!wt.infinite)
            for (int i = tid; i < kBuckets; i += kThreads)
                if (sh.mass[i] < need && need <= (i + 1 < kBuckets ? sh.mass[i + 1] : total)) sh.index = i;
        __syncthreads();
        const int border = sh.index;
        int n = kMostListed + 1;
        u64 inside = 0;
        if (!wt.infinite) {
            inside = need - sh.mass[border];
            __syncthreads();
            row.all([&](uint4 v, int piece, int round) {
                u64 c = 0;
                row.each(v, piece, [&](float x, int i) {
                    const int b = x > -INFINITY ? bucket(x) : kBuckets;
                    bool take = false;
                    if (b <= border) {
                        const u64 w = wt(x);
                        take = b == border && w > 0;
                        c += b < border && w >= least ? w : 0;
                    }
                    put(sh, take, x, i);
                });
                c = wave_sum(c);
                if (lane == 0) sh.seg[round * kWaves + wave] = c;
            });
            __syncthreads();
            n = (int)sh.listed;
        }
        if (n <= kMostListed) {
            sort_list(sh, n);
            if (tid == 0) sh.index = 0;
            u64 *w = sh.mass;
            for (int i = tid; i < n; i += kThreads) w[i] = wt(listed(sh.list[i]));
            __syncthreads();
            const u64 all = scan(sh, w, n);
            for (int i = tid; i < n; i += kThreads)
                if (w[i] < inside) {
                    const u64 x = (i + 1 < n ? w[i + 1] : all) - w[i];
                    atomicMax(&sh.index, i);
                    if (x >= least) atomicAdd(&sh.seg[row.segment_of((int)sh.list[i])], x);
                }
            __syncthreads();
            const u64 last = sh.list[sh.index];
            kept = Kept{listed(last), (int)last};
            summed = true;
            __syncthreads();
        } else {
            __syncthreads();
            segment_weights(sh, row, wt, 1);
            kept = select<true>(sh, row, wt, kept, needed(scan(sh, sh.seg, segs)));
        }
    }
    if (everything) segment_weights(sh, row, wt, least);
    else if (!summed) segment_sums(sh, row, measure);
    const u64 total = scan(sh, sh.seg, segs);
    const double at = floor((double)(a.draw[r]) * (double)total);
    const u64 pick = at > 0 ? min((u64)at, total - 1) : 0;
    const int token = find_in_order(sh, row, pick, measure);
    if (tid == 0) {
        a.token[r] = token;
        if (a.prob) a.prob[r] = (float)((double)wt((float)row.row[token]) / (double)total);
    }
}

}  // namespace

hipError_t launch_sample(const SampleArgs &a, int32_t type, hipStream_t s)
{
    if (type == INFAAS_SEL_TYPE_FP32) k_sample<float><<<a.rows, kThreads, 0, s>>>(a);
    else if (type == INFAAS_SEL_TYPE_BF16) k_sample<bf16_t><<<a.rows, kThreads, 0, s>>>(a);
    else k_sample<fp16_t><<<a.rows, kThreads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace infaas
