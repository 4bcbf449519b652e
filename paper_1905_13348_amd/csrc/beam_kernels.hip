// A step of beam search (infaas_sel_exec_beam): the best continuations of each row's parts, then of each query.
#include "exec.h"

#include <algorithm>
#include <type_traits>

namespace infaas {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kList = 2048;          // candidates of a part or a query that are put in order in LDS
constexpr uint32_t kNever = 0x007fffffu;     // order key of -infinity
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

// The greatest value that at least n of a wave's lanes reach, with its lower 16 bits cut off (0: there are not so many).
__device__ __forceinline__ uint32_t reached_by(uint32_t key, int n)
{
    uint32_t t = 0;
#pragma unroll
    for (int bit = 31; bit >= 16; --bit) {
        const uint32_t next = t | 1u << bit;
        if ((int)__popcll(__ballot(key >= next)) >= n) t = next;
    }
    return t;
}

constexpr int kWaveList = kList / kWaves;

struct PartShared {
    u64 list[kList];
    uint32_t bound[kWaves];
    float top[kWaves];
    double sum[kWaves];
    int counts[kWaves];
};

// ---- parts --------------------------------------------------------------------------------------

// A workgroup takes a part of a row, whose logits stay in registers: one read of memory for the maximum, the sum of weights and
// the best ones.  A thread's logits go by their numbers, not by addresses (its loads of 16 bytes are aligned to a logit only), so
// rows with the same logits have the same sum wherever they begin.
template <typename T, int PIECES> struct Part {
    static constexpr int E = 16 / sizeof(T), COUNT = E * PIECES, SIZE = kThreads * COUNT;
    static_assert(COUNT <= 32, "");
};
typedef vec<uint32_t, 4> Piece;
typedef Piece PieceAt2 __attribute__((aligned(2)));
typedef Piece PieceAt4 __attribute__((aligned(4)));

template <typename T, int PIECES>
__global__ __launch_bounds__(kThreads) void k_beam_parts(BeamArgs a)
{
    typedef Part<T, PIECES> P;
    typedef std::conditional_t<sizeof(T) == 2, PieceAt2, PieceAt4> Unaligned;
    constexpr int E = P::E;
    __shared__ PartShared sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t all = (int64_t)a.queries * a.beams * a.parts;
    for (int64_t g = blockIdx.x; g < all; g += gridDim.x) {
        const int row = (int)(g / a.parts), part = (int)(g % a.parts);
        if (!alive(a, row) || ended(a, row)) continue;
        const T *const logits = (const T *)a.logits + row * a.row_stride;
        const int first = part * P::SIZE;
        auto index = [&](int i) { return first + (i / E * kThreads + tid) * E + i % E; };
        float x[P::COUNT];
#pragma unroll
        for (int j = 0; j < PIECES; ++j) {
            T y[E];
            const int i0 = index(j * E);
            if (i0 + E <= a.vocab) {
                const Piece v = *(const Unaligned *)(logits + i0);
                __builtin_memcpy(y, &v, 16);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) y[e] = i0 + e < a.vocab ? logits[i0 + e] : (T)-INFINITY;
            }
#pragma unroll
            for (int e = 0; e < E; ++e) x[j * E + e] = (float)y[e];
        }

        float top, most[PIECES];
        double total;
        uint32_t least;
        while (true) {
            float mine = -INFINITY;
#pragma unroll
            for (int j = 0; j < PIECES; ++j) {
                most[j] = x[j * E];
#pragma unroll
                for (int e = 1; e < E; ++e) most[j] = fmaxf(most[j], x[j * E + e]);
                mine = fmaxf(mine, most[j]);
            }
            top = wave_max(mine);
            // of a wave alone so many lanes have one at least as great: the part's best are not below any wave's bound
            const uint32_t bound = reached_by(mine > -INFINITY ? key_of(mine) : 0, a.picks);
            __syncthreads();
            if (lane == 0) { sh.top[wave] = top; sh.bound[wave] = bound; }
            __syncthreads();
            top = fmaxf(fmaxf(sh.top[0], sh.top[1]), fmaxf(sh.top[2], sh.top[3]));
            least = max(max(max(sh.bound[0], sh.bound[1]), max(sh.bound[2], sh.bound[3])), kNever + 1);
            // Weights in 32 bits, a thread's up to 32 added there by pieces (ten roundings at the most), the threads' in 64.
            const float off = top > -INFINITY ? top : 0.0f;
            float sum = 0;
#pragma unroll
            for (int j = 0; j < PIECES; ++j) {
                float w[E];
#pragma unroll
                for (int e = 0; e < E; ++e)
                    w[e] = __builtin_amdgcn_exp2f((x[j * E + e] - off) * 1.44269504088896f);
#pragma unroll
                for (int n = E / 2; n; n /= 2)
#pragma unroll
                    for (int e = 0; e < n; ++e) w[e] += w[e + n];
                sum += w[0];
            }
            if (top == INFINITY) {      // (then the exponents were none)
                sum = 0;
#pragma unroll
                for (int i = 0; i < P::COUNT; ++i) sum += x[i] == top ? 1.0f : 0.0f;
            }
            const double wave_total = wave_sum(mine == mine ? sum : NAN);
            if (lane == 0) sh.sum[wave] = wave_total;
            __syncthreads();
            total = sh.sum[0] + sh.sum[1] + sh.sum[2] + sh.sum[3];
            if (total == total) break;
            // There are logits that are no numbers: they are taken out, once.
#pragma unroll
            for (int i = 0; i < P::COUNT; ++i) x[i] = x[i] > -INFINITY ? x[i] : -INFINITY;
        }

        // Each wave lists what reaches the bound.
        const float from = value_of(least);
        int mine_listed = 0;
        auto put = [&](bool is, float z, int i) {
            const u64 who = __ballot(is);
            if (!who) return;
            const int at = mine_listed + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0));
            if (is && at < kWaveList) sh.list[wave * kWaveList + at] = (u64)key_of(z) << 32 | (uint32_t)~index(i);
            mine_listed += (int)__popcll(who);
        };
#pragma unroll
        for (int j = 0; j < PIECES; ++j) {
            if (!__any(most[j] >= from)) continue;
#pragma unroll
            for (int e = 0; e < E; ++e) put(x[j * E + e] >= from, x[j * E + e], j * E + e);
        }
        if (lane == 0) sh.counts[wave] = mine_listed;
        __syncthreads();
        if (max(max(sh.counts[0], sh.counts[1]), max(sh.counts[2], sh.counts[3])) > kWaveList) {
            // Too many reach the bound (equal ones, mostly): the value of the last that is wanted, bit by bit over all threads, and of
            // those with that value the ones with the lowest numbers.
            uint32_t t = 0;
            for (int bit = 31; bit >= 0; --bit) {
                const uint32_t next = t | 1u << bit;
                int n = 0;
#pragma unroll
                for (int i = 0; i < P::COUNT; ++i) n += key_of(x[i]) >= next;
                for (int d = 1; d < 64; d <<= 1) n += __shfl_xor(n, d);
                __syncthreads();
                if (lane == 0) sh.counts[wave] = n;
                __syncthreads();
                if (sh.counts[0] + sh.counts[1] + sh.counts[2] + sh.counts[3] >= a.picks) t = next;
            }
            mine_listed = 0;
            int taken = 0;      // of the pieces of one number, the threads in order
            for (int j = 0; j < PIECES; ++j) {
                int mine_at = 0;
#pragma unroll
                for (int i = 0; i < P::COUNT; ++i) mine_at += i / E == j && key_of(x[i]) == t;
                int inc = mine_at;
                for (int d = 1; d < 64; d <<= 1) {
                    const int o = __shfl_up(inc, d);
                    if (lane >= d) inc += o;
                }
                __syncthreads();
                if (lane == 63) sh.counts[wave] = inc;
                __syncthreads();
                int at = taken + inc - mine_at;
                for (int w = 0; w < kWaves; ++w) {
                    if (w < wave) at += sh.counts[w];
                    taken += sh.counts[w];
                }
#pragma unroll
                for (int i = 0; i < P::COUNT; ++i)
                    if (i / E == j) put(key_of(x[i]) > t || (key_of(x[i]) == t && at++ < a.picks), x[i], i);
            }
            __syncthreads();
            if (lane == 0) sh.counts[wave] = mine_listed;
            __syncthreads();
        }
        // In order: an entry's place is the number of greater ones.  (First all of a query's parts' firsts, then their seconds.)  Four threads to an entry, one for each wave's list.
        const int ends[kWaves] = {sh.counts[0], sh.counts[0] + sh.counts[1], sh.counts[0] + sh.counts[1] + sh.counts[2],
                                  sh.counts[0] + sh.counts[1] + sh.counts[2] + sh.counts[3]};
        const int n = ends[kWaves - 1], lists = a.beams * a.parts;
        u64 *const best = a.best + g / lists * lists * a.picks + g % lists;
        for (int i0 = 0; i0 < n; i0 += kThreads / kWaves) {
            const int i = i0 + tid / kWaves, l = tid % kWaves;
            const int w = (i >= ends[0]) + (i >= ends[1]) + (i >= ends[2]);
            const u64 entry = i < n ? sh.list[w * kWaveList + i - (w ? ends[w - 1] : 0)] : ~0ull;
            int before = 0;
            const int to = sh.counts[l];
#pragma unroll 4
            for (int j = 0; j < to; ++j) before += sh.list[l * kWaveList + j] > entry;
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
    u64 wave_rank[kQueryWaves], wave_number[kQueryWaves];
};

// A workgroup takes a query: the sums of its rows' parts, and of all parts' best the best.  A row to a wave, an entry to a
// thread, which comes while the sums are computed.  (With 256 threads, and entries looked up again in every pass, 24 queries of 8
// beams of 13 parts took 25 us.)
__global__ __launch_bounds__(kQueryThreads) void k_beam_queries(BeamArgs a)
{
    __shared__ QueryShared sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int lists = a.beams * a.parts;
    const int64_t listed = (int64_t)lists * a.picks;
    for (int q = blockIdx.x; q < a.queries; q += gridDim.x) {
        const u64 *const best = a.best + q * listed;
        const u64 held = tid < listed ? best[tid] : 0;
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
        auto from_list = [&](int64_t i, u64 e, double &rank, u64 &number) {
            if (e == 0) return false;
            const int w = (int)((uint32_t)(i % lists) / (uint32_t)a.parts);
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
            for (int64_t i = tid; i < listed; i += kQueryThreads) {
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
        const uint32_t bound = reached_by(mine, a.picks);
        if (lane == 0) sh.bound[wave] = bound;
        __syncthreads();
        uint32_t least = 0;
        for (int w = 0; w < kQueryWaves; ++w) least = max(least, sh.bound[w]);
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

// Logits of a part: 8192, or 2048 where those would make too few workgroups.
constexpr int kLarge = 8192, kSmall = 2048, kFewParts = 512;

}  // namespace

BeamSizes beam_sizes(int32_t queries, int32_t beams, int32_t vocab, int32_t picks)
{
    BeamSizes z{};
    const int64_t rows = (int64_t)queries * beams;
    z.size = rows * ((vocab + kLarge - 1) / kLarge) < kFewParts ? kSmall : kLarge;
    z.parts = (vocab + z.size - 1) / z.size;
    const int64_t groups = rows * z.parts;
    z.sum_at = groups * picks * (int64_t)sizeof(u64);
    z.top_at = z.sum_at + groups * (int64_t)sizeof(double);
    z.bytes = z.top_at + groups * (int64_t)sizeof(float);
    return z;
}

hipError_t launch_beam(const BeamArgs &a, int32_t size, int32_t type, hipStream_t s)
{
    const bool small = size == kSmall;
    switch (type) {
    case INFAAS_SEL_TYPE_FP32: return small ? beam<float, 2>(a, s) : beam<float, 8>(a, s);
    case INFAAS_SEL_TYPE_BF16: return small ? beam<bf16_t, 1>(a, s) : beam<bf16_t, 4>(a, s);
    default: return small ? beam<fp16_t, 1>(a, s) : beam<fp16_t, 4>(a, s);
    }
}

}  // namespace infaas
