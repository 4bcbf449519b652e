// A step of beam search (infaas_sel_exec_beam): the best continuations of each row's parts, then of each query.
#include "exec.h"

#include <algorithm>
#include <type_traits>

namespace infaas {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kList = 2048;          // candidates of a part or a query that are put in order in LDS
constexpr uint32_t kNever = 0x007fffffu;     // order key of -infinity
constexpr float kLog2e = 1.44269504088896f;
// Beyond it a product with log2(e) is rounded by more than 2^-12: the difference is taken first, then.
constexpr float kNear = 2048.0f;
typedef unsigned long long u64;

// Logits that are numbers as 32-bit keys in their order: equal logits (-0 and +0, too) have equal keys.
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t k) { return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k); }
__device__ __forceinline__ u64 key_of(double x)
{
    const u64 b = __double_as_longlong(x + 0.0);
    return b >> 63 ? ~b : b | 1ull << 63;
}

// A neighbour's value in the steps of a reduction over a wave: 1, 2, 4 and 8 lanes down within rows of 16, then the last lane of a
// row into the next one, and of the lower half into the upper; lanes without one get `none`.  The result is in lane 63.  (Six
// operations; through LDS each step is a trip of a hundred cycles.)
template <int CTRL, int ROWS> __device__ __forceinline__ int neighbour(int x, int none) { return __builtin_amdgcn_update_dpp(none, x, CTRL, ROWS, 0xf, false); }
template <typename F> __device__ __forceinline__ void over_wave(F step)
{
    step(std::integral_constant<int, 0x111>(), std::integral_constant<int, 0xf>());
    step(std::integral_constant<int, 0x112>(), std::integral_constant<int, 0xf>());
    step(std::integral_constant<int, 0x114>(), std::integral_constant<int, 0xf>());
    step(std::integral_constant<int, 0x118>(), std::integral_constant<int, 0xf>());
    step(std::integral_constant<int, 0x142>(), std::integral_constant<int, 0xa>());
    step(std::integral_constant<int, 0x143>(), std::integral_constant<int, 0xc>());
}
__device__ __forceinline__ float wave_max(float x)
{
    over_wave([&](auto ctrl, auto rows) { x = fmaxf(x, __int_as_float(neighbour<ctrl.value, rows.value>(__float_as_int(x), __float_as_int(-INFINITY)))); });
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}
__device__ __forceinline__ double wave_sum(double x)
{
    over_wave([&](auto ctrl, auto rows) {
        x += __hiloint2double(neighbour<ctrl.value, rows.value>(__double2hiint(x), 0), neighbour<ctrl.value, rows.value>(__double2loint(x), 0));
    });
    return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(x), 63), __builtin_amdgcn_readlane(__double2loint(x), 63));
}

// log(x) of a normal positive number: 2^e m with m from 1/sqrt(2) to sqrt(2), log m = 2 artanh z, z = (m - 1) / (m + 1), |z| <= 0.172;
// behind the term z^17 / 17 the series has 0.172^19 / 19 = 2e-16 left.  (A few lines of code: the library's takes longer to fetch
// than to run, once a launch.)
__device__ __forceinline__ double log_of(double x)
{
    int e = 0;
    double m = frexp(x, &e);
    if (m < 0.70710678118654752) { m *= 2; --e; }
    const double z = (m - 1) / (m + 1), zz = z * z;
    double p = 1.0 / 17;
#pragma unroll
    for (int n = 15; n >= 1; n -= 2) p = __builtin_fma(p, zz, 1.0 / n);
    return __builtin_fma((double)e, 0.69314718055994531, 2 * z * p);
}

// What a beam has to continue with.  Dead ones (scores that are not finite, factors that are not positive) have nothing.
__device__ __forceinline__ bool alive(const BeamArgs &a, int row)
{
    return fabsf(a.scores[row]) < INFINITY && (!a.factor || (a.factor[row] > 0 && a.factor[row] < INFINITY));
}
__device__ __forceinline__ bool ended(const BeamArgs &a, int row) { return a.ended && a.ended[row] != 0; }

// The greatest value that at least n of a wave's lanes reach, with its lower bits cut off (0: there are not so many).
template <int LOWEST> __device__ __forceinline__ uint32_t reached_by(uint32_t key, int n)
{
    uint32_t t = 0;
#pragma unroll
    for (int bit = 31; bit >= LOWEST; --bit) {
        const uint32_t next = t | 1u << bit;
        if ((int)__popcll(__ballot(key >= next)) >= n) t = next;
    }
    return t;
}

// The same of a workgroup's threads, wave by wave through `counts`.  Where many are picked: a wave alone has too few lanes then for
// a bound that is of use.  (64 picks, 16 queries of 8 beams x 128,000 fp32: with the waves' bounds 741 us, so 56.)
constexpr int kManyPicks = 16;
template <int LOWEST, int WAVES> __device__ __forceinline__ uint32_t reached_by_all(uint32_t key, int n, int (*counts)[WAVES])
{
    uint32_t t = 0;
#pragma unroll 1
    for (int bit = 31; bit >= LOWEST; --bit) {
        const uint32_t next = t | 1u << bit;
        const int mine = (int)__popcll(__ballot(key >= next));
        if ((threadIdx.x & 63) == 0) counts[bit & 1][threadIdx.x >> 6] = mine;
        __syncthreads();
        int all = 0;
        for (int w = 0; w < WAVES; ++w) all += counts[bit & 1][w];
        if (all >= n) t = next;
    }
    return t;
}

// A wave's candidates: up to kKept, and those of a piece to each lane behind them.
constexpr int kKept = 2 * kMostBeams, kWaveList = kKept + 64 * 8;

struct PartShared {
    u64 list[kWaves][kWaveList];
    uint32_t bound[kWaves];
    float top[kWaves];
    double sum[kWaves];
    int counts[kWaves], reached[2][kWaves];
};

// What all lanes' bits have in common (OF_ALL) or any lane's.
template <bool OF_ALL> __device__ __forceinline__ uint32_t bits_of_wave(uint32_t x)
{
    over_wave([&](auto ctrl, auto rows) {
        const uint32_t y = (uint32_t)neighbour<ctrl.value, rows.value>((int)x, OF_ALL ? -1 : 0);
        x = OF_ALL ? x & y : x | y;
    });
    return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}

__device__ __forceinline__ uint32_t min_of_wave(uint32_t x)
{
    over_wave([&](auto ctrl, auto rows) { x = min(x, (uint32_t)neighbour<ctrl.value, rows.value>((int)x, -1)); });
    return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}

// The n entries of a wave's list become the `want` greatest (n is more), in any order; the least of them is returned.  Bit by bit
// from the first in which entries differ, until just so many are left; where those with the least logit (a mask's) are among
// them, from the first bit in which these differ.  (Few registers and not long code: it stands in every
// piece's way.  Rows whose logits are -60,000 but for 129, 512 rows of 128,000 bf16: from the first bit in which any differ 150 us,
// so 57.)
__device__ __forceinline__ u64 keep_greatest(u64 *list, int n, int want)
{
    const int lane = threadIdx.x & 63;
    u64 both = ~0ull, any = 0;
    uint32_t lowest = ~0u;
#pragma unroll 2
    for (int i = 0; i < n; i += 64) {
        const u64 x = list[min(i + lane, n - 1)];
        both &= x;
        any |= x;
        lowest = min(lowest, (uint32_t)(x >> 32));
    }
    lowest = min_of_wave(lowest);
    int above = 0;
    for (int i = 0; i < n; i += 64) above += (int)__popcll(__ballot(i + lane < n && (uint32_t)(list[min(i + lane, n - 1)] >> 32) > lowest));
    if (above < want) {
        both = ~0ull, any = 0;
        for (int i = 0; i < n; i += 64) {
            const u64 x = list[min(i + lane, n - 1)];
            if ((uint32_t)(x >> 32) == lowest) { both &= x; any |= x; }
        }
    }
    both = (u64)bits_of_wave<true>((uint32_t)(both >> 32)) << 32 | bits_of_wave<true>((uint32_t)both);
    any = (u64)bits_of_wave<false>((uint32_t)(any >> 32)) << 32 | bits_of_wave<false>((uint32_t)any);
    int bit = 63 - __builtin_clzll(both ^ any);      // (entries differ: each has a number of its own)
    u64 t = both & ~((2ull << bit) - 1);
#pragma unroll 1
    for (; bit >= 0; --bit) {
        const u64 next = t | 1ull << bit;
        int count = 0;
        for (int i = 0; i < n; i += 64) count += (int)__popcll(__ballot(i + lane < n && list[min(i + lane, n - 1)] >= next));
        if (count >= want) t = next;
        if (count == want) break;
    }
    int at = 0;
#pragma unroll 1
    for (int i = 0; i < n; i += 64) {
        const u64 mine = i + lane < n ? list[i + lane] : 0;
        const u64 who = __ballot(mine >= t);
        if (mine >= t) list[at + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0))] = mine;
        at += (int)__popcll(who);
    }
    return t;
}

// ---- parts --------------------------------------------------------------------------------------

// A workgroup takes a part of a row, `chunks` times `PIECES` pieces of 16 bytes to a thread: one read of memory for the maximum,
// the sum of weights and the best ones.  A thread's logits go by their numbers, not by addresses (its loads of 16 bytes are
// aligned to a logit only), so rows with the same logits have the same sum wherever they begin.
// What bounds it: vector instructions, 60% of the time, and the waits between them (512 rows of 128,000 bf16, 131 MB: 36 us, 3.6 TB/s where a
// large copy reaches 5.2; fp32, twice the bytes, 58 with the queries' kernel).  Of 400 instructions a wave and chunk of 2048 logits 180 are
// the conversion, maximum, exponent and sum of each, the others bounds and lists.  (An exact sum in 64 bits of every weight 68 us; lists by
// atomics 57; a part of one chunk 42.)
typedef vec<uint32_t, 4> Piece;
typedef Piece PieceAt2 __attribute__((aligned(2)));
typedef Piece PieceAt4 __attribute__((aligned(4)));

template <typename T, int PIECES>
__global__ __launch_bounds__(kThreads, 4) void k_beam_parts(BeamArgs a)
{
    typedef std::conditional_t<sizeof(T) == 2, PieceAt2, PieceAt4> Unaligned;
    constexpr int E = 16 / sizeof(T), COUNT = E * PIECES, CHUNK = kThreads * COUNT;
    __shared__ PartShared sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    u64 *const list = sh.list[wave];
    const uint32_t all = (uint32_t)a.queries * a.beams * a.parts;
    for (uint32_t g = blockIdx.x; g < all; g += gridDim.x) {
        const int row = (int)(g / (uint32_t)a.parts), part = (int)(g % (uint32_t)a.parts);
        if (!alive(a, row) || ended(a, row)) continue;
        const T *const logits = (const T *)a.logits + row * a.row_stride;
        const int first = part * a.chunks * CHUNK, chunks = min(a.chunks, (a.vocab - first - 1) / CHUNK + 1);
        Piece raw[PIECES];
        // (a piece that goes beyond the row's end is read from so many logits earlier, and those are left out: see below)
        auto number = [&](int i0) { return min(i0, max(a.vocab - E, 0)); };
        auto load = [&](int c) {
#pragma unroll
            for (int j = 0; j < PIECES; ++j) raw[j] = *(const Unaligned *)(logits + number(first + c * CHUNK + (j * kThreads + tid) * E));
        };
        auto load_first = [&] {
            if (a.vocab >= E) return load(0);
            T y[E];
#pragma unroll
            for (int e = 0; e < E; ++e) y[e] = e < a.vocab ? logits[e] : (T)-INFINITY;
#pragma unroll
            for (int j = 0; j < PIECES; ++j) __builtin_memcpy(&raw[j], y, 16);
        };
        float top;
        double total;
        int listed;
        // What kind of numbers there are shows in the sum: kind 0 takes the logits as they come, 1 takes out what is no number, 2
        // counts those of +infinity (the weights of the others are 0).
        for (int kind = 0;; ++kind) {
            // A lane's greatest, and the wave's, which weights are taken against: its product with log2(e), rounded, and what the
            // rounding makes of a weight, to the first power.  (One operation for each exponent, and no error but its own rounding.)
            float mine = -INFINITY, ref = 0, halvings = 0;
            double correction = 1;
            double sum = 0;
            uint32_t least = 0;
            float from = 0;
            listed = 0;
            load_first();
            for (int c = 0; c < chunks; ++c) {
                float x[COUNT], most[PIECES];
#pragma unroll
                for (int j = 0; j < PIECES; ++j) {
                    T y[E];
                    __builtin_memcpy(y, &raw[j], 16);
#pragma unroll
                    for (int e = 0; e < E; ++e) x[j * E + e] = (float)y[e];
                    const int i0 = first + c * CHUNK + (j * kThreads + tid) * E;
                    if (i0 + E > a.vocab) {
#pragma unroll
                        for (int e = 0; e < E; ++e) x[j * E + e] = number(i0) + e >= i0 ? x[j * E + e] : -INFINITY;
                    }
                }
                if (c + 1 < chunks) load(c + 1);
                if (kind)
#pragma unroll
                    for (int i = 0; i < COUNT; ++i) x[i] = x[i] > -INFINITY ? x[i] : -INFINITY;
#pragma unroll
                for (int j = 0; j < PIECES; ++j) {
                    most[j] = x[j * E];
#pragma unroll
                    for (int e = 1; e < E; ++e) most[j] = fmaxf(most[j], x[j * E + e]);
                    mine = fmaxf(mine, most[j]);
                }
                // of a wave alone so many lanes have one at least as great: the part's best are not below any wave's bound
                const uint32_t key = mine > -INFINITY ? key_of(mine) : 0;
                if (a.picks <= kManyPicks || c) least = max(least, reached_by<16>(key, a.picks));
                if (c == 0 && a.picks > kManyPicks) {
                    least = max(reached_by_all<16, kWaves>(key, a.picks, sh.reached), kNever + 1);
                } else if (c == 0) {
                    __syncthreads();
                    if (lane == 0) sh.bound[wave] = least;
                    __syncthreads();
                    least = max(max(max(sh.bound[0], sh.bound[1]), max(sh.bound[2], sh.bound[3])), kNever + 1);
                }
                from = value_of(least);
                top = wave_max(mine);
                const float now = top > -INFINITY ? top : 0.0f;
                if (kind < 2 && now != ref) {
                    // (nothing as yet stays nothing: the first reference can be far below 0)
                    sum = sum > 0 ? sum * (double)__builtin_amdgcn_exp2f((ref - now) * 1.44269504088896f) : sum;
                    ref = now;
                    halvings = ref * kLog2e;
                    correction = 1 + ((double)halvings - (double)ref * (double)kLog2e) * 0.69314718055994531;
                }
                // Weights in 32 bits, a chunk's up to 32 added there by pieces (ten roundings at the most), all others in 64.
                auto add_up = [&](auto weight) {
                    float all_pieces = 0;
#pragma unroll
                    for (int j = 0; j < PIECES; ++j) {
                        float w[E];
#pragma unroll
                        for (int e = 0; e < E; ++e) w[e] = weight(x[j * E + e]);
#pragma unroll
                        for (int n = E / 2; n; n /= 2)
#pragma unroll
                            for (int e = 0; e < n; ++e) w[e] += w[e + n];
                        all_pieces += w[0];
                    }
                    return all_pieces;
                };
                if (kind < 2 && fabsf(ref) < kNear) {
                    const float part_sum = add_up([&](float z) { return __builtin_amdgcn_exp2f(__builtin_fmaf(z, kLog2e, -halvings)); });
                    sum = __builtin_fma((double)part_sum, correction, sum);
                } else if (kind < 2) {
                    sum += (double)add_up([&](float z) { return __builtin_amdgcn_exp2f((z - ref) * kLog2e); });
                } else {
                    sum += (double)add_up([&](float z) { return z == INFINITY ? 1.0f : 0.0f; });
                }
                // Each wave lists what reaches the bound, group by group in the logits' order.
#pragma unroll
                for (int j = 0; j < PIECES; ++j) {
                    if (!__any(most[j] >= from)) continue;
                    if (listed > kKept) {      // then only what is greater than all but the kept ones counts: equal ones come later
                        least = max(least, (uint32_t)(keep_greatest(list, listed, a.picks) >> 32) + 1);
                        from = value_of(least);
                        listed = a.picks;
                    }
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const bool is = x[j * E + e] >= from;
                        const u64 who = __ballot(is);
                        if (!who) continue;
                        const int at = listed + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0));
                        if (is) list[at] = (u64)key_of(x[j * E + e]) << 32 | (uint32_t)~(number(first + c * CHUNK + (j * kThreads + tid) * E) + e);
                        listed += (int)__popcll(who);
                    }
                }
            }
            if (listed > kKept) {
                keep_greatest(list, listed, a.picks);
                listed = a.picks;
            }
            const double wave_total = wave_sum(mine == mine ? sum : NAN);
            if (lane == 0) {
                sh.top[wave] = top;
                sh.sum[wave] = wave_total;
                sh.counts[wave] = listed;
            }
            __syncthreads();
            top = fmaxf(fmaxf(sh.top[0], sh.top[1]), fmaxf(sh.top[2], sh.top[3]));
            total = 0;
            for (int w = 0; w < kWaves; ++w)
                total += kind == 2 || sh.top[w] == top ? sh.sum[w] : sh.sum[w] * (double)__builtin_amdgcn_exp2f((sh.top[w] - top) * 1.44269504088896f);
            if (kind == 2 || fabs(total) < INFINITY) break;
        }
        // In order: an entry's place is the number of greater ones.  (First all of a query's parts' firsts, then their seconds.)  Four
        // threads to an entry, one for each wave's list.
        const int ends[kWaves] = {sh.counts[0], sh.counts[0] + sh.counts[1], sh.counts[0] + sh.counts[1] + sh.counts[2],
                                  sh.counts[0] + sh.counts[1] + sh.counts[2] + sh.counts[3]};
        const int n = ends[kWaves - 1], lists = a.beams * a.parts;
        u64 *const best = a.best + (int64_t)(g / (uint32_t)lists) * lists * a.picks + g % (uint32_t)lists;
        for (int i0 = 0; i0 < n; i0 += kThreads / kWaves) {
            const int i = i0 + tid / kWaves, l = tid % kWaves;
            const int w = (i >= ends[0]) + (i >= ends[1]) + (i >= ends[2]);
            const u64 entry = i < n ? sh.list[w][i - (w ? ends[w - 1] : 0)] : ~0ull;
            int before = 0;
            const int to = sh.counts[l];
#pragma unroll 4
            for (int j = 0; j < to; ++j) before += sh.list[l][j] > entry;
            before += __shfl_xor(before, 1);
            before += __shfl_xor(before, 2);
            if (i < n && l == 0 && before < a.picks) best[(int64_t)before * lists] = entry;
        }
        for (int i = n + tid; i < a.picks; i += kThreads) best[(int64_t)i * lists] = 0;
        if (tid == 0) {
            a.top[g] = top;
            a.sum[g] = total;
        }
    }
}

// ---- queries ------------------------------------------------------------------------------------

constexpr int kQueryThreads = 1024, kQueryWaves = kQueryThreads / 64;

struct QueryShared {
    double rank[kList];
    u64 number[kList];       // beam * 2^32 + token
    // of every beam: what its greatest logit scores (NaN: its parts have no candidates), what it scores itself (NaN: it has not
    // ended), its factor, its greatest logit
    double shift[kMostBeams], score[kMostBeams], factor[kMostBeams];
    float top[kMostBeams];
    uint32_t listed, bound[kQueryWaves];
    int reached[2][kQueryWaves];
    u64 wave_rank[kQueryWaves], wave_number[kQueryWaves];
};

// A workgroup takes a query: the sums of its rows' parts, and of all parts' best the best.  A row to a wave, an entry to a
// thread, which comes while the sums are computed.  (With 256 threads, and entries looked up again in every pass, 24 queries of 8
// beams of 13 parts took 25 us, so 11; 128 queries of 4 beams of 4 parts 6.)
__global__ __launch_bounds__(kQueryThreads) void k_beam_queries(BeamArgs a)
{
    __shared__ QueryShared sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t lists = a.beams * a.parts, listed = lists * a.picks;      // (2^21 at the most)
    for (int q = blockIdx.x; q < a.queries; q += gridDim.x) {
        const u64 *const best = a.best + (int64_t)q * listed;
        const u64 held = (uint32_t)tid < listed ? best[tid] : 0;
        __syncthreads();
        for (int w = wave; w < a.beams; w += kQueryWaves) {
            const int row = q * a.beams + w;
            const float *const tops = a.top + (int64_t)row * a.parts;
            const double *const sums = a.sum + (int64_t)row * a.parts;
            // (everything that may be needed is under way at once)
            const float t0 = lane < a.parts ? tops[lane] : -INFINITY;
            const double s0 = lane < a.parts ? sums[lane] : 0.0;
            const double own = a.scores[row], factor = a.factor ? a.factor[row] : 1.0;
            const bool is_alive = alive(a, row), is_ended = ended(a, row);
            double shift = NAN;
            float top = t0;
            for (int p = lane + 64; p < a.parts; p += 64) top = fmaxf(top, tops[p]);
            top = wave_max(top);
            auto weight = [&](float t) {
                return t == top ? 1.0 : t > -INFINITY && top < INFINITY ? (double)__builtin_amdgcn_exp2f((t - top) * 1.44269504088896f) : 0.0;
            };
            double sum = weight(t0) * s0;
            for (int p = lane + 64; p < a.parts; p += 64) sum += weight(tops[p]) * sums[p];
            sum = wave_sum(sum);
            if (is_alive && !is_ended && top > -INFINITY) shift = own - log_of(sum);
            if (lane == 0) {
                sh.shift[w] = shift;
                sh.score[w] = is_alive && is_ended ? own : NAN;
                sh.factor[w] = factor;
                sh.top[w] = top;
            }
        }
        if (tid == 0) sh.listed = 0;
        __syncthreads();
        // rank and number of an entry of the parts' lists, if it is a candidate
        auto from_list = [&](uint32_t i, u64 e, double &rank, u64 &number) {
            if (e == 0) return false;
            const int w = (int)(i % lists / (uint32_t)a.parts);
            const double shift = sh.shift[w];
            const float x = value_of((uint32_t)(e >> 32)), top = sh.top[w];
            if (!(shift == shift) || (top == INFINITY && x < top)) return false;
            rank = (x == top ? shift : shift + ((double)x - (double)top)) * sh.factor[w];
            number = (u64)w << 32 | (uint32_t)~e;
            return true;
        };
        // f(rank, number) of all candidates: the held ones, those beyond them, the beams that have ended
        auto each = [&](auto f) {
            double rank;
            u64 number;
            u64 e = held;
#pragma unroll 1
            for (uint32_t i = tid; i < listed; i += kQueryThreads) {
                if (from_list(i, e, rank, number)) f(rank, number);
                if (i + kQueryThreads < listed) e = best[i + kQueryThreads];
            }
            if (tid < a.beams) {      // (the arrays are not looked at again: the result may be one of them)
                const double score = sh.score[tid];
                if (score == score) f(score * sh.factor[tid], (u64)tid << 32 | (uint32_t)a.end_token);
            }
        };
        uint32_t mine = 0;
        each([&](double rank, u64) { mine = max(mine, (uint32_t)(key_of(rank) >> 32)); });
        uint32_t least = 0;      // (to 12 bits behind the first: 11 are the exponent's)
        if (a.picks <= kManyPicks) {
            const uint32_t bound = reached_by<8>(mine, a.picks);
            if (lane == 0) sh.bound[wave] = bound;
            __syncthreads();
            for (int w = 0; w < kQueryWaves; ++w) least = max(least, sh.bound[w]);
        } else {
            least = reached_by_all<8, kQueryWaves>(mine, a.picks, sh.reached);
        }
        each([&](double rank, u64 number) {
            if ((uint32_t)(key_of(rank) >> 32) < least) return;
            const uint32_t at = atomicAdd(&sh.listed, 1u);
            if (at < kList) { sh.rank[at] = rank; sh.number[at] = number; }
        });
        __syncthreads();
        const int64_t out = (int64_t)q * a.picks;
        auto write = [&](int place, double rank, u64 number) {
            const int w = (int)(number >> 32);
            a.out_parent[out + place] = q * a.beams + w;
            a.out_token[out + place] = (int)(uint32_t)number;
            a.out_score[out + place] = a.factor ? (float)(rank / sh.factor[w]) : (float)rank;
        };
        int found = (int)sh.listed;
        if (found <= kList) {
            for (int i = tid; i < found; i += kQueryThreads) {
                const double rank = sh.rank[i];
                const u64 number = sh.number[i];
                int before = 0;
#pragma unroll 4
                for (int j = 0; j < found; ++j) before += sh.rank[j] > rank || (sh.rank[j] == rank && sh.number[j] < number);
                if (before < a.picks) write(before, rank, number);
            }
        } else {
            // More than the list holds share the bound: one after the other, each the first behind the one before it.
            double last = INFINITY;
            u64 last_number = 0;
            for (found = 0; found < a.picks; ++found) {
                u64 most = 0, which = ~0ull;
                each([&](double rank, u64 number) {
                    if (!(rank < last || (rank == last && found > 0 && number > last_number))) return;
                    const u64 k = key_of(rank);
                    if (k > most || (k == most && number < which)) { most = k; which = number; }
                });
                for (int d = 1; d < 64; d <<= 1) {
                    const u64 k = __shfl_xor(most, d), n = __shfl_xor(which, d);
                    if (k > most || (k == most && n < which)) { most = k; which = n; }
                }
                __syncthreads();
                if (lane == 0) { sh.wave_rank[wave] = most; sh.wave_number[wave] = which; }
                __syncthreads();
                most = 0, which = ~0ull;
                for (int w = 0; w < kQueryWaves; ++w)
                    if (sh.wave_rank[w] > most || (sh.wave_rank[w] == most && sh.wave_number[w] < which)) { most = sh.wave_rank[w]; which = sh.wave_number[w]; }
                if (most == 0) break;
                last = __longlong_as_double(most >> 63 ? most & ~(1ull << 63) : ~most);
                last_number = which;
                if (tid == 0) write(found, last, last_number);
            }
        }
        for (int i = found + tid; i < a.picks; i += kQueryThreads) {
            a.out_parent[out + i] = a.out_token[out + i] = -1;
            a.out_score[out + i] = -INFINITY;
        }
    }
}

template <typename T, int PIECES> hipError_t beam(const BeamArgs &a, hipStream_t s)
{
    const int64_t groups = (int64_t)a.queries * a.beams * a.parts;
    k_beam_parts<T, PIECES><<<(unsigned)std::min<int64_t>(groups, 1 << 20), kThreads, 0, s>>>(a);
    if (hipError_t e = hipGetLastError()) return e;
    k_beam_queries<<<std::min(a.queries, 1 << 16), kQueryThreads, 0, s>>>(a);
    return hipGetLastError();
}

// Logits of a chunk: 8192, or 2048 where those would make too few workgroups; a part has several chunks where there are many
// rows, since what a part costs besides is that of about 8192 logits.
constexpr int kLarge = 8192, kSmall = 2048, kFewParts = 512, kManyParts = 2048, kMostChunks = 4;

}  // namespace

BeamSizes beam_sizes(int32_t queries, int32_t beams, int32_t vocab, int32_t picks)
{
    BeamSizes z{};
    const int64_t rows = (int64_t)queries * beams;
    const int64_t large = rows * ((vocab + kLarge - 1) / kLarge);
    z.chunk = large < kFewParts ? kSmall : kLarge;
    z.chunks = std::max<int64_t>(1, std::min<int64_t>(kMostChunks, large / kManyParts));
    z.parts = (vocab + z.chunk * z.chunks - 1) / (z.chunk * z.chunks);
    const int64_t groups = rows * z.parts;
    z.sum_at = groups * picks * (int64_t)sizeof(u64);
    z.top_at = z.sum_at + groups * (int64_t)sizeof(double);
    z.bytes = z.top_at + groups * (int64_t)sizeof(float);
    return z;
}

hipError_t launch_beam(const BeamArgs &a, const BeamSizes &z, int32_t type, hipStream_t s)
{
    const bool small = z.chunk == kSmall;
    switch (type) {
    case INFAAS_SEL_TYPE_FP32: return small ? beam<float, 2>(a, s) : beam<float, 8>(a, s);
    case INFAAS_SEL_TYPE_BF16: return small ? beam<bf16_t, 1>(a, s) : beam<bf16_t, 4>(a, s);
    default: return small ? beam<fp16_t, 1>(a, s) : beam<fp16_t, 4>(a, s);
    }
}

}  // namespace infaas
