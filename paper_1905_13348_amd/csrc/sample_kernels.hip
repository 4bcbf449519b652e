// Drawing a token of every row of logits (infaas_sel_exec_sample).
#include "exec.h"

#include <algorithm>
#include <type_traits>

namespace infaas {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kSegment = 1024;               // tokens of a row whose weights are summed by a wave at a time
constexpr int kMostSegments = 1025;          // 2^20 logits at any alignment
constexpr int kMostListed = 2048;            // candidates that are put in order in LDS, two to a thread
constexpr int kBuckets = 2048;               // of logits by their distance from the greatest
constexpr int kShift = 43;                   // a weight of 1 is 2^43: 2^20 of them stay below 2^63
constexpr float kFar = 44.0f;                // in halvings: weights further down are 0 units
constexpr float kNone = 45.0f;               // ... also as computed
constexpr uint32_t kNever = 0x007fffffu;     // order key of -infinity
constexpr int kLastIndex = 0x7fffffff;
// Loops that run once a row are not unrolled: the first fetch of instructions costs hundreds of cycles per 64 bytes, and one
// row with all limits is done in the time of a few such fetches (16 rounds of the bound's search unrolled: 10 us).
constexpr unsigned long long kRaw = 0x4330000000000000ull;   // the bits of 2^52

typedef unsigned long long u64;

// Bins of bf16 logits, one for each of the values from 2^-12 to 2^7 of either sign, the least first, and one between the
// signs for everything that is nearer to zero.
constexpr int kBinLow = 115 << 7;            // the bits of 2^-12
constexpr int kBinSide = 19 << 7;            // values of one sign
constexpr int kTinyBin = kBinSide, kBins = 2 * kBinSide + 1;
constexpr float kBinEnd = 128.0f;
constexpr int kMostTiny = 2048;
// Shorter rows are not counted by value: to clear the bins and to sum them up takes as long as what is gained.
constexpr int kLeastBinned = 4096;

// Logits that are numbers as 32-bit keys in their order: equal logits (-0 and +0, too) have equal keys.
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t k) { return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k); }

// (ln 2)^n / n!, n = 0 .. 11.
__constant__ double kSeries[12] = {1.0, 0.69314718055994531, 0.24022650695910072, 0.055504108664821580, 0.0096181291076284772,
                                   0.0013333558146428443, 1.5403530393381610e-4, 1.5252733804059840e-5, 1.3215486790144309e-6,
                                   1.0178086009239699e-7, 7.0549116208011233e-9, 4.4455382718708116e-10};

// 2^(43 + j/128), for the table of a workgroup: the Taylor series of e^(f ln 2), |f| <= 1/2, to the eleventh power (what is
// left out is 0.347^12 / 12! = 6e-15 of it).
constexpr int kPowers = 128;
__device__ double power_of(int j)
{
    const double f = (j < kPowers / 2 ? j : j - kPowers) * (1.0 / kPowers);
    double p = kSeries[11];
#pragma unroll 1
    for (int i = 10; i >= 0; --i) p = __builtin_fma(p, f, kSeries[i]);
    return p * (j < kPowers / 2 ? (double)(1ull << kShift) : (double)(2ull << kShift));
}

// Weights exp((x - top) / temperature) in units of 2^-43: 2^t, t = (x - top) * log2(e) / temperature, as 2^(n/128) from the
// table times the Taylor series of 2^(f/128) = e^(f ln 2 / 128), |f| <= 1/2, to the fourth power: what is left out is
// 0.0027^5 / 5! = 1e-15 of it.  (Operations on doubles take twice the time of others; the series to the eleventh power
// instead of the table 10% more for a pass over 256 x 128,000 logits.)
struct Weights {
    double top, per, c[5];      // per: 128 log2(e) / temperature
    const double *powers;
    __device__ __forceinline__ void init(const double *table, float greatest, float temperature)
    {
        powers = table;
        top = greatest == INFINITY ? 1e300 : (double)greatest;      // (of what is finite then nothing is left)
        per = greatest == INFINITY ? 1e300 : 1.4426950408889634 * kPowers / (double)temperature;
        double scale = 1.0;
#pragma unroll
        for (int i = 0; i < 5; ++i, scale *= 1.0 / kPowers) c[i] = kSeries[i] * scale;
    }
    __device__ __forceinline__ double halvings() const { return per * (1.0 / kPowers); }      // to a logit's unit
    // The units plus kRaw (for sums of many: one subtraction at the end instead of one each).  A weight is rounded to units
    // by adding 2^52 to the double, whose bits are then those of the units behind the exponent; t below the range gives 0.
    __device__ __forceinline__ u64 raw(float x) const
    {
        // (NaN, of a logit or of 0 times infinity, becomes the lower end, infinity 0)
        const double t = fmin(fmax(((double)x - top) * per, -(double)kNone * kPowers), 0.0);
        constexpr double whole = 6755399441055744.0;      // 1.5 * 2^52: adding it rounds to an integer, in the low bits
        const double r = t + whole, f = t - (r - whole);
        const int n = (int)__double_as_longlong(r);
        double p = c[4];
#pragma unroll
        for (int i = 3; i >= 0; --i) p = __builtin_fma(p, f, c[i]);
        const u64 scaled = __double_as_longlong(p * powers[n & (kPowers - 1)]) + ((u64)(uint32_t)(n >> 7) << 52);
        return __double_as_longlong(__longlong_as_double(scaled) + 4503599627370496.0);
    }
    __device__ __forceinline__ u64 operator()(float x) const { return raw(x) - kRaw; }
};
static_assert(kPowers == 1 << 7, "");

// What is kept: everything above `value`, and of the tokens at it those numbered up to `last`.  (Never NaN.)
struct Kept {
    float value;
    int last;
    __device__ __forceinline__ bool has(float x, int i) const { return x > value || (x == value && i <= last); }
};

struct Shared {
    u64 seg[kMostSegments];
    union {
        u64 list[kMostListed];
        uint32_t count_of[kBins];
    };
    u64 mass[kBins];      // (or kBuckets of them; of kMostListed weights)
    uint32_t count[256];
    int tiny[kMostTiny];
    uint32_t wave_count[kWaves];
    struct { int bin; u64 kept, before; } border;
    uint32_t far;

    u64 wave_sum[kWaves];
    u64 digits[16];
    double powers[kPowers];
    float wave_top[kWaves];
    uint32_t listed;
    int index;
    u64 left;
};

__device__ __forceinline__ u64 wave_sum(u64 v)
{
#pragma unroll 1
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// A row in pieces of 16 bytes, at the addresses that are multiples of 16.  A wave takes segments of 1024 tokens, the waves
// of the workgroup segments side by side; a piece per lane at a time, so that a pass's code is that of a few tokens (a
// long unrolled body costs more in fetches of instructions than it saves).
template <typename T>
struct Row {
    typedef T Type;
    static constexpr int E = 16 / sizeof(T), DEEP = kSegment / (64 * E), AHEAD = 4;
    const T *row;
    int V, shift, last, segments, whole0, whole1;      // segments whole0 .. whole1-1 lie within the row altogether

    __device__ __forceinline__ void init(const T *p, int n)
    {
        row = p;
        V = n;
        shift = (int)((uintptr_t)p / sizeof(T) % E);
        last = (V + shift - 1) / E * E - shift;
        segments = (V + shift + kSegment - 1) / kSegment;
        whole0 = shift ? 1 : 0;
        whole1 = max(whole0, (V + shift) / kSegment);
    }
    __device__ __forceinline__ int segment_of(int i) const { return (i + shift) / kSegment; }
    // the token that a lane's piece begins with; pieces are numbered by segment and place in it
    __device__ __forceinline__ int first(int piece) const { return (piece * 64 + (int)(threadIdx.x & 63)) * E - shift; }
    // (A piece that the row begins or ends in is read whole: its 16 bytes are on one page with a token's.)
    __device__ __forceinline__ uint4 read(int piece) const { return *(const uint4 *)(row + min(first(piece), last)); }
    // f(logit, token) of every token of a piece; what is no token counts as -infinity, NaN may come
    template <typename F> __device__ __forceinline__ void each(uint4 v, int piece, F f) const
    {
        T x[E];
        __builtin_memcpy(x, &v, 16);
        const int seg = piece / DEEP, i = first(piece);
        if (seg < whole0 || seg >= whole1)
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = i + e >= 0 && i + e < V ? x[e] : (T)-INFINITY;
#pragma unroll
        for (int e = 0; e < E; ++e) f((float)x[e], i + e);
    }
    // f(word, upper half) of every token of a piece of 16 bits each, by bits; what is no token counts as -infinity
    template <typename F> __device__ __forceinline__ void each_bits(uint4 v, int piece, F f) const
    {
        static_assert(std::is_same<T, bf16_t>::value, "");
        uint32_t w[4] = {v.x, v.y, v.z, v.w};
        const int seg = piece / DEEP, i = first(piece);
        if (seg < whole0 || seg >= whole1)
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (i + e < 0 || i + e >= V) w[e / 2] = e % 2 ? (w[e / 2] & 0xffff) | 0xff800000u : (w[e / 2] & 0xffff0000u) | 0xff80;
#pragma unroll
        for (int e = 0; e < E; ++e) f(w[e / 2], e % 2 != 0);
    }
    // body(piece's contents, its number) for all pieces, and ended(segment) behind the last of each segment.  Four pieces are
    // worked on, one after the other, while the next four are under way; they change places all at once, because a
    // register that a load is under way to cannot be moved.
    template <typename F, typename G> __device__ __forceinline__ void all(F body, G ended) const
    {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int mine = wave < segments ? ((segments - 1 - wave) / kWaves + 1) * DEEP : 0;      // pieces of this wave
        auto number = [&](int j) { return (wave + j / DEEP * kWaves) * DEEP + j % DEEP; };
        if (mine == 0) return;
        uint4 now[AHEAD], next[AHEAD];
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) next[a] = read(number(min(a, mine - 1)));
#pragma unroll 1
        for (int j0 = 0; j0 < mine; j0 += AHEAD) {
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) now[a] = next[a];
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) next[a] = read(number(min(j0 + AHEAD + a, mine - 1)));
            const int to = min(AHEAD, mine - j0);
#pragma unroll 1
            for (int a = 0; a < to; ++a) {
                const uint4 lo = a & 1 ? now[1] : now[0], hi = a & 1 ? now[3] : now[2];
                body(a & 2 ? hi : lo, number(j0 + a));
                if ((j0 + a) % DEEP == DEEP - 1) ended(number(j0 + a) / DEEP);
            }
        }
    }
    template <typename F> __device__ __forceinline__ void all(F body) const { all(body, [](int) {}); }
};

// Running sums over v[0 .. n-1] in place (each entry: what is in front of it); returns the total.  All threads.
__device__ u64 scan(Shared &sh, u64 *v, int n)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, each = (n + kThreads - 1) / kThreads;
    u64 sum = 0;
#pragma unroll 1
    for (int i = tid * each; i < min(n, (tid + 1) * each); ++i) sum += v[i];
    u64 inc = sum;
#pragma unroll 1
    for (int d = 1; d < 64; d <<= 1) {
        const u64 o = __shfl_up(inc, d);
        if (lane >= d) inc += o;
    }
    if (lane == 63) sh.wave_sum[wave] = inc;
    __syncthreads();
    u64 before = inc - sum, all = 0;
#pragma unroll 1
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) before += sh.wave_sum[w];
        all += sh.wave_sum[w];
    }
#pragma unroll 1
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
    u64 c = 0;
    row.all([&](uint4 v, int piece) { row.each(v, piece, [&](float x, int i) { c += f(x, i); }); },
            [&](int seg) {
                c = wave_sum(c);
                if ((threadIdx.x & 63) == 0) sh.seg[seg] = c;
                c = 0;
            });
    __syncthreads();
}

// The same of all weights.
template <typename R> __device__ __forceinline__ void segment_weights(Shared &sh, R &row, const Weights &wt)
{
    u64 c = 0;
    row.all([&](uint4 v, int piece) { row.each(v, piece, [&](float x, int) { c += wt.raw(x); }); },
            [&](int seg) {
                c = wave_sum(c - (kSegment / 64) * kRaw);
                if ((threadIdx.x & 63) == 0) sh.seg[seg] = c;
                c = 0;
            });
    __syncthreads();
}

// The token whose measure f(logit, token), added to those of the tokens with lower numbers, first exceeds `at` (which is
// less than the sum of all).  `sums` are the running sums of the segments.  All threads get the answer.
template <typename R, typename F> __device__ int find_in_order(Shared &sh, R &row, const u64 *sums, u64 at, F f)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, segs = row.segments;
#pragma unroll 1
    for (int i = tid; i < segs; i += kThreads) {
        const u64 next = i + 1 < segs ? sums[i + 1] : ~0ull;
        if (sums[i] <= at && at < next) sh.index = i;      // (of segments that add nothing the last: one thread)
    }
    __syncthreads();
    const int seg = sh.index, i = seg * kSegment + tid - row.shift;      // a token to a thread
    static_assert(kSegment == kThreads, "");
    const u64 w = i >= 0 && i < row.V ? f((float)row.row[i], i) : 0;
    u64 inc = w;
#pragma unroll 1
    for (int d = 1; d < 64; d <<= 1) {
        const u64 o = __shfl_up(inc, d);
        if (lane >= d) inc += o;
    }
    if (lane == 63) sh.wave_sum[wave] = inc;
    __syncthreads();
    inc += sums[seg];
#pragma unroll 1
    for (int v = 0; v < wave; ++v) inc += sh.wave_sum[v];
    if (inc - w <= at && at < inc) sh.index = i;             // (one thread)
    __syncthreads();
    return sh.index;
}

// The next place of a counter, for every lane that asks: one atomic for all of them.
__device__ __forceinline__ uint32_t next_place(uint32_t *counter)
{
    const u64 mask = __ballot(1);
    uint32_t base = 0;
    const int before = __popcll(mask & ((1ull << (threadIdx.x & 63)) - 1));
    if (before == 0) base = atomicAdd(counter, (uint32_t)__popcll(mask));
    return __builtin_amdgcn_readfirstlane(base) + before;
}

// Adds (logit, token) to sh.list; counts on beyond the list's end.
__device__ __forceinline__ void put(Shared &sh, float x, int i)
{
    const uint32_t at = next_place(&sh.listed);
    if (at < kMostListed) sh.list[at] = (u64)~key_of(x) << 32 | (uint32_t)i;
}

// Puts the n entries of sh.list in order, the greatest logit first, equal ones by number.  Up to kThreads of them each find
// their place by counting those in front of it, which takes three barriers instead of one for each step of the sort; several
// threads share an entry's count.  (With a shorter search for the bound: one row of 32,768 fp32 with all limits 26 us, so 22.)
__device__ void sort_list(Shared &sh, int n)
{
    const int tid = threadIdx.x;
    int m = 64;
    while (m < n) m *= 2;
#pragma unroll 1
    for (int i = n + tid; i < m; i += kThreads) sh.list[i] = ~0ull;
    if (m <= kThreads) {
        sh.tiny[tid] = 0;
        __syncthreads();
        const int entry = tid & (m - 1), part = tid / m, each = m / (kThreads / m);
        const u64 mine = sh.list[entry];
        int before = 0;
#pragma unroll 4
        for (int j = 0; j < each; ++j) before += sh.list[part * each + j] < mine;
        if (before) atomicAdd(&sh.tiny[entry], before);
        __syncthreads();
        if (tid < n) sh.list[sh.tiny[tid]] = mine;
        __syncthreads();
        return;
    }
    __syncthreads();
#pragma unroll 1
    for (int size = 2; size <= m; size *= 2)
#pragma unroll 1
        for (int step = size / 2; step; step /= 2) {
            const int i = (tid / step) * step * 2 + tid % step, j = i + step;
            const bool up = (i & size) == 0;
            const u64 x = sh.list[i], y = sh.list[j];
            if ((x > y) == up) { sh.list[i] = y; sh.list[j] = x; }
            __syncthreads();
        }
}
static_assert(kMostListed == 2 * kThreads && kMostTiny >= kThreads, "");
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
#pragma unroll 1
        for (int i = tid; i < 256; i += kThreads) sh.count[i] = 0, sh.mass[i] = 0;
        __syncthreads();
        const uint32_t mask = shift == 24 ? 0u : ~0u << (shift + 8);
        row.all([&](uint4 v, int piece) {
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
    scan(sh, sh.seg, row.segments);
    return Kept{value, find_in_order(sh, row, sh.seg, m - 1, is)};
}

// Units in front of which a token is still kept.
__device__ __forceinline__ u64 needed(float top_p, u64 total)
{
    const double need = ceil((double)top_p * (double)total);
    return need >= 1.0 ? (u64)need : 1ull;
}

// Rows of bf16: 128,000 logits have a few thousand values.  They are counted by value, weighted once to a value, and the
// borders of all limits are found among the values; a second pass looks the weights up.  Neither pass computes an
// exponential, and the first needs no maximum in front of it.  For top-p alone and for a top-k that the list is too short
// for: 512 x 128,000 with top-p 221 us by buckets of weights, so 110; one row of 4096 18.3, so 15.6.  (A top-k that fits
// the list is done sooner by it: 64 x 128,000 34 us, by bins 53; without limits the passes cost as much as the weights.)
// Returns false (all threads do) where that is not enough: logits of 128 and more, a border or the maximum among those near
// zero, or too many of these.  Otherwise `wt` and `kept` are set and sh.seg has the sums of what is kept, by segments.
// Nothing is expected of sh.
template <typename R>
__device__ bool by_bins(Shared &sh, R &row, Weights &wt, Kept &kept, float temperature, int k, bool by_k, float top_p, bool by_p,
                        u64 least)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    uint32_t *const count = sh.count_of;
    constexpr int MINE = (kBins + kThreads - 1) / kThreads;      // bins of a thread
    auto place = [](float x) { return (int)(__float_as_uint(x) >> 16 & 0x7fff) - kBinLow; };      // among those of its sign
    // bin of a logit by its bits, kTinyBin + 1 .. or kTinyBin - 1 .. by its place; whether there is one
    auto bin_by = [](uint32_t word, bool upper, int &bin) {
        const int d = (int)((upper ? word >> 16 : word) & 0x7fff) - (kBinLow - 1), sign = (int)(upper ? word : word << 16) >> 31;
        bin = kTinyBin + ((d ^ sign) - sign);
        return (uint32_t)(d - 1) < (uint32_t)kBinSide;
    };
    auto value = [](int bin) {
        const int d = bin < kTinyBin ? kBinSide - 1 - bin : bin - kBinSide - 1;
        return __uint_as_float((uint32_t)(d + kBinLow) << 16 | (bin < kTinyBin ? 0x80000000u : 0u));
    };
#pragma unroll 1
    for (int i = tid; i < kBins; i += kThreads) count[i] = 0;
    if (tid == 0) { sh.listed = 0; sh.far = 0; sh.index = kBins; sh.left = 0; sh.border.bin = -1; }
    __syncthreads();
    uint32_t far = 0;
    row.all([&](uint4 v, int piece) {
        bool odd = false;
        row.each_bits(v, piece, [&](uint32_t word, bool upper) {
            int bin;
            const bool in = bin_by(word, upper, bin);
            if (in) atomicAdd(&count[bin], 1u);
            odd |= !in;
        });
        if (__any(odd))
            row.each(v, piece, [&](float x, int i) {
                const int d = place(x);
                if (d < 0) {
                    const uint32_t at = next_place(&sh.listed);
                    if (at < kMostTiny) sh.tiny[at] = i;
                } else if (d >= kBinSide) {
                    far |= x >= kBinEnd ? 1u : x > -INFINITY ? 2u : 0u;      // (NaN and -infinity: neither)
                }
            });
    });
    if (far) atomicOr(&sh.far, far);
    __syncthreads();
    const int tiny = (int)sh.listed;
    far = sh.far;
    // some bins to a thread, the greatest first
    auto bin_of = [&](int j) { return kBins - 1 - (MINE * tid + j); };
    uint32_t c[MINE];
    int first = kBins;
#pragma unroll
    for (int j = MINE - 1; j >= 0; --j) {
        const int bin = bin_of(j);
        c[j] = bin < 0 ? 0 : bin == kTinyBin ? (uint32_t)tiny : count[bin];
        if (c[j]) first = kBins - 1 - bin;
    }
    if (first < kBins) atomicMin(&sh.index, first);
    __syncthreads();
    const int top_bin = kBins - 1 - sh.index;
    if (top_bin < 0 || top_bin == kTinyBin || tiny > kMostTiny || (far & 1)) return false;
    wt.init(sh.powers, value(top_bin), temperature);
    // (what is below the bins has no weight, or is more than the bins can tell)
    if ((far & 2) && ((double)-kBinEnd - wt.top) * wt.halvings() > -(double)kNone) return false;
    u64 w[MINE], mass[MINE], m = 0, tiny_mass = 0;
#pragma unroll 1
    for (int i = tid; i < tiny; i += kThreads) tiny_mass += wt((float)row.row[sh.tiny[i]]);
    if (tiny_mass) atomicAdd(&sh.left, tiny_mass);
#pragma unroll
    for (int j = 0; j < MINE; ++j) w[j] = c[j] && bin_of(j) != kTinyBin ? wt(value(bin_of(j))) : 0;
    __syncthreads();
    uint32_t n = 0;
#pragma unroll
    for (int j = 0; j < MINE; ++j) {
        mass[j] = bin_of(j) == kTinyBin ? sh.left : c[j] * w[j];
        m += mass[j];
        n += c[j];
    }
    u64 sum_m = m;
    uint32_t sum_n = n;
#pragma unroll 1
    for (int d = 1; d < 64; d <<= 1) {
        const u64 om = __shfl_up(sum_m, d);
        const uint32_t on = __shfl_up(sum_n, d);
        if (lane >= d) { sum_m += om; sum_n += on; }
    }
    if (lane == 63) { sh.wave_sum[wave] = sum_m; sh.wave_count[wave] = sum_n; }
    __syncthreads();
    u64 before_m = sum_m - m, total = 0;
    uint32_t before_n = sum_n - n;
#pragma unroll 1
    for (int v = 0; v < kWaves; ++v) {
        if (v < wave) { before_m += sh.wave_sum[v]; before_n += sh.wave_count[v]; }
        total += sh.wave_sum[v];
    }
    if (by_k) {      // the bin in which the k-th token is, and how many of its tokens are among the k
        u64 bm = before_m;
        uint32_t bn = before_n;
#pragma unroll
        for (int j = 0; j < MINE; ++j) {
            if (bn < (uint32_t)k && (uint32_t)k <= bn + c[j]) { sh.border = {bin_of(j), (uint32_t)k - bn, bm + ((uint32_t)k - bn) * w[j]}; }
            bm += mass[j];
            bn += c[j];
        }
        __syncthreads();
        if (sh.border.bin == kTinyBin) return false;
        if (sh.border.bin >= 0) total = sh.border.before;
    }
    if (by_p) {      // the same of the token at which the weights reach what is needed
        const u64 need = needed(top_p, total);
        u64 bm = before_m;
        if (by_k) __syncthreads();      // (everybody has read the first border)
#pragma unroll
        for (int j = 0; j < MINE; ++j) {
            if (bm < need && need <= bm + mass[j]) sh.border = {bin_of(j), w[j] ? (need - bm + w[j] - 1) / w[j] : 0, 0};
            bm += mass[j];
        }
        __syncthreads();
        if (sh.border.bin == kTinyBin) return false;
    }
    const int bin = sh.border.bin;
    const u64 of_bin = sh.border.kept, weight = bin >= 0 ? wt(value(bin)) : 0;
    const bool ties = bin >= 0 && of_bin < count[bin];
    constexpr int kTieShift = 48;           // a lane's sixteen tokens of a segment weigh less
    static_assert(kSegment / 64 * 2 <= 1 << (kTieShift - kShift), "");
#pragma unroll
    for (int j = 0; j < MINE; ++j) {
        const int b = bin_of(j);
        if (b >= 0) sh.mass[b] = b == bin && ties ? 1ull << kTieShift : b < bin || b == kTinyBin || w[j] < least ? 0 : w[j];
    }
    __syncthreads();
    u64 *const tie_count = sh.list;         // (the counts have been read)
    u64 sum = 0;
    row.all([&](uint4 v, int piece) {
                row.each_bits(v, piece, [&](uint32_t word, bool upper) {
                    int bin;
                    const bool in = bin_by(word, upper, bin);
                    sum += sh.mass[in ? bin : kTinyBin];
                });
            },
            [&](int seg) {
                const u64 s = wave_sum(sum & ((1ull << kTieShift) - 1));
                if (ties) {
                    const u64 t = wave_sum(sum >> kTieShift);
                    if (lane == 0) tie_count[seg] = t;
                }
                if (lane == 0) sh.seg[seg] = s;
                sum = 0;
            });
    __syncthreads();
    if (bin < kTinyBin)
#pragma unroll 1
        for (int i = tid; i < tiny; i += kThreads) {
            const u64 x = wt((float)row.row[sh.tiny[i]]);
            if (x >= least) atomicAdd(&sh.seg[row.segment_of(sh.tiny[i])], x);
        }
    if (bin >= 0) kept = Kept{value(bin), kLastIndex};
    if (ties) {
        const float at = kept.value;
        const int segs = row.segments;
        const u64 all = scan(sh, tie_count, segs);      // (begins and ends with a barrier)
        kept.last = find_in_order(sh, row, tie_count, of_bin - 1, [&](float x, int) -> u64 { return x == at; });
        if (weight >= least)
#pragma unroll 1
            for (int i = tid; i < segs; i += kThreads) {
                const u64 here = tie_count[i], next = i + 1 < segs ? tie_count[i + 1] : all;
                if (here < of_bin) sh.seg[i] += (min(next, of_bin) - here) * weight;
            }
    }
    __syncthreads();
    return true;
}

// A workgroup per row: the greatest logit, then what is kept, by whichever way is short for the row's limits, with the
// sums of its weights by segments, then the segment that the draw falls into.
//   top-k up to kThreads: the k-th of the threads' greatest logits is a bound that k tokens at least reach; those are
//     listed, put in order, and cut by all limits there.  For small k they are few more than k.  From some 85% of the threads
//     that hold tokens on (64 for each 1024 tokens, up to 1024) the list is too short, and what follows comes on top:
//     one row of 128,000 with a top-k of 200 31 us, 832 53, 896 to 1024 212 in bf16 (1025, by value, 52).
//   top-p alone: of bf16 by value (by_bins); else weights summed into buckets of logits; the bucket that the border is in is
//     listed and put in order.
//   neither: nothing to find.
// Where the lists are too short (top-k near and above kThreads, thousands of equal logits at a border) the border is found eight
// bits at a time (one row of 128,000 fp32 or fp16 with a top-k of 1025: 170 us).
// What bounds it: passes over a row by one compute unit (two at least: what is kept goes by the greatest, or by what is
// counted), which holds one workgroup (94 to 106 registers) and so has nothing else to do at a row's barriers and ends.
// 256 x 128,000 fp32 without limits 60 us: vector instructions take 61% of the busy compute units' time, the waves wait for
// 43% of theirs.  512 x 128,000 bf16 with top-p 110 (two rounds, 0.23 ns a token and row): 69%, and LDS 40%, half of that
// conflicts; fp16 200 and fp32 218, by buckets.  One row of 32,768 fp32 with all limits 22, where every pass waits for its
// loads and each new piece of code for its instructions.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_sample(SampleArgs a, int first)
{
    __shared__ Shared sh;
    const int r = first + blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), V = a.vocab;
    Row<T> row;
    row.init((const T *)a.logits + r * a.row_stride, V);
    const int segs = row.segments;
    const float t = a.temperature ? a.temperature[r] : 1.0f;
    const float top_p = a.top_p ? a.top_p[r] : 1.0f, min_p = a.min_p && a.min_p[r] > 0 ? a.min_p[r] : 0.0f;
    const bool greedy = !(t > 0) || min_p > 1.0f;
    const int k = a.top_k ? a.top_k[r] : 0;

    // the least weight that is kept, in units: w >= min_p as numbers is rint(2^43 w) >= this but for what is nearer to the
    // border than half a unit
    const u64 least = max((u64)rint((double)min_p * (double)(1ull << kShift)), 1ull);
    const bool by_p = top_p < 1.0f, by_k = k > 0 && k < V;
    Weights wt;
    Kept kept{-INFINITY, -1};            // everything
    auto measure = [&](float x, int i) -> u64 {
        const u64 w = wt(x);
        return kept.has(x, i) && w >= least ? w : 0;
    };
    if (tid < kPowers) sh.powers[tid] = power_of(tid);      // (a barrier comes before the first weight)
    bool done = false;
    if constexpr (std::is_same<T, bf16_t>::value)
        if (!greedy && (by_k ? k > kThreads : by_p) && V >= kLeastBinned) {
            done = by_bins(sh, row, wt, kept, t, k, by_k, top_p, by_p, least);
            __syncthreads();
        }
    if (!done) {
        if (tid < 16) sh.digits[tid] = 0;
        if (tid == 0) { sh.listed = 0; sh.index = kLastIndex; }
        float mine = -INFINITY;
        int at_token = kLastIndex;
        if (greedy) row.all([&](uint4 v, int piece) { row.each(v, piece, [&](float x, int i) { if (x > mine) { mine = x; at_token = i; } }); });
        else row.all([&](uint4 v, int piece) { row.each(v, piece, [&](float x, int) { mine = fmaxf(mine, x); }); });
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
        wt.init(sh.powers, top, t);
        // The list holds the tokens among which the last that is kept is, and sh.seg the sums of those that are kept for sure.
        // In the list `inside` units or, if that is 0, what top_p makes of the first k.
        int n = kMostListed + 1;
        u64 inside = 0;
        if (by_k && k <= kThreads) {
            // the k-th greatest of the threads' greatest, two bits at a time, or a little less: its first eighteen
            uint32_t bound = 0;
            const uint32_t mine_key = key_of(mine);
#pragma unroll 1
            for (int bit = 30; bit >= 14; bit -= 2) {
                u64 c = 0;
#pragma unroll
                for (int d = 1; d < 4; ++d) c |= (u64)__popcll(__ballot(mine_key >= (bound | (uint32_t)d << bit))) << (16 * d);
                if (lane == 0) atomicAdd(&sh.digits[bit / 2], c);
                __syncthreads();
                c = sh.digits[bit / 2];
                const uint32_t d = ((c >> 16 & 0xffff) >= (u64)k) + ((c >> 32 & 0xffff) >= (u64)k) + ((c >> 48) >= (u64)k);
                bound |= d << bit;
            }
            // (a bound of no number: fewer threads than k have logits at all)
            const float from = bound <= kNever ? -INFINITY : value_of(bound);
            row.all([&](uint4 v, int piece) { row.each(v, piece, [&](float x, int i) { if (x >= from && x > -INFINITY) put(sh, x, i); }); });
#pragma unroll 1
            for (int s = tid; s < segs; s += kThreads) sh.seg[s] = 0;
            __syncthreads();
            n = (int)sh.listed;
        } else if (by_p && !by_k && top < INFINITY) {
            const float per = fminf((float)(wt.halvings() * (kBuckets / (double)kFar)), 3e38f);
            auto bucket = [&](float x) { return (int)fminf((top - x) * per, (float)(kBuckets - 1)); };
#pragma unroll 1
            for (int i = tid; i < kBuckets; i += kThreads) sh.mass[i] = 0;
            __syncthreads();
            row.all([&](uint4 v, int piece) {
                row.each(v, piece, [&](float x, int) {
                    const u64 w = wt(x);
                    if (w) atomicAdd(&sh.mass[bucket(x)], w);
                });
            });
            __syncthreads();
            const u64 total = scan(sh, sh.mass, kBuckets), need = needed(top_p, total);
#pragma unroll 1
            for (int i = tid; i < kBuckets; i += kThreads)
                if (sh.mass[i] < need && need <= (i + 1 < kBuckets ? sh.mass[i + 1] : total)) sh.index = i;
            __syncthreads();
            const int border = sh.index;
            inside = need - sh.mass[border];
            segment_sums(sh, row, [&](float x, int i) -> u64 {
                const int b = x > -INFINITY ? bucket(x) : kBuckets;
                if (b > border) return 0;
                const u64 w = wt(x);
                if (b == border && w > 0) put(sh, x, i);
                return b < border && w >= least ? w : 0;
            });
            n = (int)sh.listed;
        }

        if (n <= kMostListed) {
            sort_list(sh, n);
            if (tid == 0) sh.index = 0;
            u64 *w = sh.mass;                // (as many entries as the list)
            const int most = inside ? n : min(k, n);
#pragma unroll 1
            for (int i = tid; i < n; i += kThreads) w[i] = i < most ? wt(listed(sh.list[i])) : 0;
            __syncthreads();
            const u64 all = scan(sh, w, n), need = inside ? inside : by_p ? needed(top_p, all) : ~0ull;
#pragma unroll 1
            for (int i = tid; i < most; i += kThreads) {
                const u64 x = (i + 1 < n ? w[i + 1] : all) - w[i];
                if (w[i] < need) {
                    atomicMax(&sh.index, i);
                    if (x >= least) atomicAdd(&sh.seg[row.segment_of((int)sh.list[i])], x);
                }
            }
            __syncthreads();
            const u64 last = sh.list[sh.index];
            kept = Kept{listed(last), (int)last};
            __syncthreads();
        } else {
            if (by_k) kept = select<false>(sh, row, wt, kept, (u64)k);
            if (by_p) {
                segment_sums(sh, row, [&](float x, int i) -> u64 { return kept.has(x, i) ? wt(x) : 0; });
                kept = select<true>(sh, row, wt, kept, needed(top_p, scan(sh, sh.seg, segs)));
            }
            if (by_k || by_p || least > 1) segment_sums(sh, row, measure);
            else segment_weights(sh, row, wt);
        }
    }
    const u64 total = scan(sh, sh.seg, segs);
    const double at = floor((double)(a.draw[r]) * (double)total);
    const u64 pick = at > 0 ? min((u64)at, total - 1) : 0;
    const int token = find_in_order(sh, row, sh.seg, pick, measure);
    if (tid == 0) {
        a.token[r] = token;
        if (a.prob) a.prob[r] = (float)((double)wt((float)row.row[token]) / (double)total);
    }
}

}  // namespace

hipError_t launch_sample(const SampleArgs &a, int32_t type, hipStream_t s)
{
    for (int64_t first = 0; first < a.rows; first += kMostGroups) {
        const dim3 grid((unsigned)std::min(kMostGroups, a.rows - first));
        if (type == INFAAS_SEL_TYPE_FP32) k_sample<float><<<grid, kThreads, 0, s>>>(a, (int)first);
        else if (type == INFAAS_SEL_TYPE_BF16) k_sample<bf16_t><<<grid, kThreads, 0, s>>>(a, (int)first);
        else k_sample<fp16_t><<<grid, kThreads, 0, s>>>(a, (int)first);
        if (hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}

}  // namespace infaas
