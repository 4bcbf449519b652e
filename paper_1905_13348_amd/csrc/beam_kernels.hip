// A step of beam search (infaas_sel_exec_beam): the best continuations of each row's parts, then of each query.
#include "exec.h"

#include <algorithm>

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

// Puts the n entries of a list in order: f(place, entry) for each, from the greatest key.
template <typename F> __device__ __forceinline__ void in_order(const u64 *list, int n, int want, F f)
{
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const u64 mine = list[i];
        int before = 0;
        for (int j = 0; j < n; ++j) before += list[j] > mine;
        if (before < want) f(before, mine);
    }
}

struct PartShared {
    u64 list[kList];
    uint32_t listed, bound[kWaves];
    float top[kWaves];
    double sum[kWaves];
    u64 counts[kWaves][2];
};

// ---- parts --------------------------------------------------------------------------------------

// A workgroup takes a part of a row: `kThreads * PIECES` pieces of 16 bytes less one, so that wherever the row begins the part
// lies within as many pieces at addresses that are multiples of 16.  Its logits stay in registers: one read of memory for the
// maximum, the sum of weights and the best ones.
// Weights exp(x - maximum) are rounded to multiples of 2^-40, of which 64 bits sum up 2^13 exactly: the sum does not depend on
// which thread has which logit, and rows with the same logits have the same, wherever they begin.
template <typename T, int PIECES> struct Part {
    static constexpr int E = 16 / sizeof(T), COUNT = E * PIECES, SIZE = kThreads * COUNT - E;
    static_assert(kThreads * COUNT <= 8192, "");
};

template <typename T, int PIECES>
__global__ __launch_bounds__(kThreads) void k_beam_parts(BeamArgs a)
{
    typedef Part<T, PIECES> P;
    constexpr int E = P::E;
    __shared__ PartShared sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t all = (int64_t)a.queries * a.beams * a.parts;
    for (int64_t g = blockIdx.x; g < all; g += gridDim.x) {
        const int row = (int)(g / a.parts), part = (int)(g % a.parts);
        if (!alive(a, row) || ended(a, row)) continue;
        const T *const logits = (const T *)a.logits + row * a.row_stride;
        const int first = part * P::SIZE, last = min(a.vocab, first + P::SIZE);      // (of the part)
        const int shift = (int)((uintptr_t)(logits + first) / sizeof(T) % E);
        float x[P::COUNT];
#pragma unroll
        for (int j = 0; j < PIECES; ++j) {
            const int i0 = first - shift + (j * kThreads + tid) * E;
            T y[E];
            uint4 v = uint4{};
            // (a piece that the part begins or ends in is read whole: its 16 bytes are on one page with a logit's)
            if (i0 < last) v = *(const uint4 *)(logits + i0);
            __builtin_memcpy(y, &v, 16);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float z = (float)y[e];
                x[j * E + e] = i0 + e >= first && i0 + e < last && z > -INFINITY ? z : -INFINITY;
            }
        }
        auto index = [&](int i) { return first - shift + (i / E * kThreads + tid) * E + i % E; };

        float mine = x[0];
#pragma unroll
        for (int i = 1; i < P::COUNT; ++i) mine = fmaxf(mine, x[i]);
        float top = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
        // of a wave alone so many lanes have one at least as great: the part's best are not below any wave's bound
        const uint32_t bound = reached_by(mine > -INFINITY ? key_of(mine) : 0, a.picks);
        __syncthreads();
        if (lane == 0) { sh.top[wave] = top; sh.bound[wave] = bound; }
        if (tid == 0) sh.listed = 0;
        __syncthreads();
        top = fmaxf(fmaxf(sh.top[0], sh.top[1]), fmaxf(sh.top[2], sh.top[3]));
        const uint32_t least = max(max(max(sh.bound[0], sh.bound[1]), max(sh.bound[2], sh.bound[3])), kNever + 1);

        double sum = 0;
        if (top < INFINITY) {
            constexpr float whole = 1.5f / (1 << 17);      // adding it rounds to multiples of 2^-40, or to a float's own bits
            const float off = top > -INFINITY ? top : 0.0f;
#pragma unroll
            for (int i = 0; i < P::COUNT; ++i) {
                const float w = __builtin_amdgcn_exp2f((x[i] - off) * 1.44269504088896f);
                sum += (double)((w + whole) - whole);
            }
        } else {
#pragma unroll
            for (int i = 0; i < P::COUNT; ++i) sum += x[i] == INFINITY ? 1.0 : 0.0;
        }
        for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);

        int above = 0;
#pragma unroll
        for (int i = 0; i < P::COUNT; ++i) above += key_of(x[i]) >= least;
        for (int d = 1; d < 64; d <<= 1) above += __shfl_xor(above, d);
        if (lane == 0) { sh.sum[wave] = sum; sh.counts[wave][0] = above; }
        __syncthreads();
        const u64 total = sh.counts[0][0] + sh.counts[1][0] + sh.counts[2][0] + sh.counts[3][0];
        auto put = [&](int i) {
            const uint32_t at = atomicAdd(&sh.listed, 1u);
            if (at < kList) sh.list[at] = (u64)key_of(x[i]) << 32 | (uint32_t)~index(i);
        };
        if (total <= kList) {
#pragma unroll
            for (int i = 0; i < P::COUNT; ++i)
                if (key_of(x[i]) >= least) put(i);
        } else {
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
                if (lane == 0) sh.counts[wave][0] = n;
                __syncthreads();
                if (sh.counts[0][0] + sh.counts[1][0] + sh.counts[2][0] + sh.counts[3][0] >= (u64)a.picks) t = next;
            }
            int mine_at = 0;      // of the pieces of one number, the threads in order
            uint32_t taken = 0;
            for (int j = 0; j < PIECES; ++j) {
                mine_at = 0;
#pragma unroll
                for (int i = 0; i < P::COUNT; ++i) mine_at += i / E == j && key_of(x[i]) == t;
                int inc = mine_at;
                for (int d = 1; d < 64; d <<= 1) {
                    const int o = __shfl_up(inc, d);
                    if (lane >= d) inc += o;
                }
                __syncthreads();
                if (lane == 63) sh.counts[wave][0] = inc;
                __syncthreads();
                uint32_t at = taken + inc - mine_at;
                for (int w = 0; w < kWaves; ++w) {
                    if (w < wave) at += (uint32_t)sh.counts[w][0];
                    taken += (uint32_t)sh.counts[w][0];
                }
#pragma unroll
                for (int i = 0; i < P::COUNT; ++i) {
                    if (i / E != j) continue;
                    if (key_of(x[i]) > t) put(i);
                    else if (key_of(x[i]) == t && at++ < (uint32_t)a.picks) put(i);
                }
            }
        }
        __syncthreads();
        const int n = min((int)sh.listed, kList);
        u64 *const out = a.best + g * a.picks;
        in_order(sh.list, n, a.picks, [&](int place, u64 entry) { out[place] = entry; });
        for (int i = n + tid; i < a.picks; i += kThreads) out[i] = 0;
        if (tid == 0) {
            a.top[g] = top;
            a.sum[g] = sh.sum[0] + sh.sum[1] + sh.sum[2] + sh.sum[3];
        }
    }
}

// ---- queries ------------------------------------------------------------------------------------

struct Candidate { double rank; u64 number; };      // number: beam * 2^32 + token

struct QueryShared {
    double rank[kList];
    u64 number[kList];
    // of every beam: what its greatest logit scores (NaN: its parts have no candidates), what it scores itself (NaN: it has not
    // ended), its factor, its greatest logit
    double shift[kMostBeams], score[kMostBeams], factor[kMostBeams];
    float top[kMostBeams];
    uint32_t listed, bound[kWaves];
    u64 wave_rank[kWaves], wave_number[kWaves];
};

// A workgroup takes a query: the sums of its rows' parts, and of all parts' best the best.
__global__ __launch_bounds__(kThreads) void k_beam_queries(BeamArgs a)
{
    __shared__ QueryShared sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t per_row = (int64_t)a.parts * a.picks, entries = per_row * a.beams + a.beams;
    for (int q = blockIdx.x; q < a.queries; q += gridDim.x) {
        __syncthreads();
        for (int w = wave; w < a.beams; w += kWaves) {
            const int row = q * a.beams + w;
            double shift = NAN, score = NAN, factor = 1.0;
            float top = -INFINITY;
            if (alive(a, row)) {
                if (a.factor) factor = a.factor[row];
                if (ended(a, row)) {
                    score = a.scores[row];
                } else {
                    for (int p = lane; p < a.parts; p += 64) top = fmaxf(top, a.top[(int64_t)row * a.parts + p]);
                    for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
                    double sum = 0;
                    for (int p = lane; p < a.parts; p += 64) {
                        const float t = a.top[(int64_t)row * a.parts + p];
                        const double s = a.sum[(int64_t)row * a.parts + p];
                        sum += t == top ? s : t > -INFINITY && top < INFINITY ? s * exp((double)t - (double)top) : 0.0;
                    }
                    for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
                    if (top > -INFINITY) shift = (double)a.scores[row] - log(sum);
                }
            }
            if (lane == 0) { sh.shift[w] = shift; sh.score[w] = score; sh.factor[w] = factor; sh.top[w] = top; }
        }
        if (tid == 0) sh.listed = 0;
        __syncthreads();
        // candidate i: of the parts' lists, then of the beams that have ended; false: there is none
        auto candidate = [&](int64_t i, Candidate &c, double &score) {
            if (i < entries - a.beams) {
                const int w = (int)(i / per_row);
                const u64 e = a.best[(int64_t)q * a.beams * per_row + i];
                const double shift = sh.shift[w];
                if (!(shift == shift) || e == 0) return false;
                const float x = value_of((uint32_t)(e >> 32)), top = sh.top[w];
                if (top == INFINITY && x < top) return false;
                score = x == top ? shift : shift + ((double)x - (double)top);
                c.rank = score * sh.factor[w];
                c.number = (u64)w << 32 | (uint32_t)~e;
                return true;
            }
            const int w = (int)(i - (entries - a.beams));      // (the arrays are not looked at again: the result may be one of them)
            score = sh.score[w];
            if (!(score == score)) return false;
            c.rank = score * sh.factor[w];
            c.number = (u64)w << 32 | (uint32_t)a.end_token;
            return true;
        };
        uint32_t mine = 0;
        for (int64_t i = tid; i < entries; i += kThreads) {
            Candidate c;
            double s;
            if (candidate(i, c, s)) mine = max(mine, (uint32_t)(key_of(c.rank) >> 32));
        }
        const uint32_t bound = reached_by(mine, a.picks);
        if (lane == 0) sh.bound[wave] = bound;
        __syncthreads();
        const uint32_t least = max(max(sh.bound[0], sh.bound[1]), max(sh.bound[2], sh.bound[3]));
        for (int64_t i = tid; i < entries; i += kThreads) {
            Candidate c;
            double s;
            if (!candidate(i, c, s) || (uint32_t)(key_of(c.rank) >> 32) < least) continue;
            const uint32_t at = atomicAdd(&sh.listed, 1u);
            if (at < kList) { sh.rank[at] = c.rank; sh.number[at] = c.number; }
        }
        __syncthreads();
        const int64_t out = (int64_t)q * a.picks;
        auto write = [&](int place, double rank, u64 number) {
            const int w = (int)(number >> 32), row = q * a.beams + w;
            a.out_parent[out + place] = row;
            a.out_token[out + place] = (int)(uint32_t)number;
            a.out_score[out + place] = a.factor ? (float)(rank / sh.factor[w]) : (float)rank;
        };
        int found = (int)sh.listed;
        if (found <= kList) {
            for (int i = tid; i < found; i += kThreads) {
                const double rank = sh.rank[i];
                const u64 number = sh.number[i];
                int before = 0;
                for (int j = 0; j < found; ++j) before += sh.rank[j] > rank || (sh.rank[j] == rank && sh.number[j] < number);
                if (before < a.picks) write(before, rank, number);
            }
        } else {
            // More than the list holds share the bound: one after the other, each the first behind the one before it.
            double rank = INFINITY;
            u64 number = 0;
            found = 0;
            for (; found < a.picks; ++found) {
                u64 best = 0, which = ~0ull;
                for (int64_t i = tid; i < entries; i += kThreads) {
                    Candidate c;
                    double s;
                    if (!candidate(i, c, s) || !(c.rank < rank || (c.rank == rank && found > 0 && c.number > number))) continue;
                    const u64 k = key_of(c.rank);
                    if (k > best || (k == best && c.number < which)) { best = k; which = c.number; }
                }
                for (int d = 1; d < 64; d <<= 1) {
                    const u64 k = __shfl_xor(best, d), n = __shfl_xor(which, d);
                    if (k > best || (k == best && n < which)) { best = k; which = n; }
                }
                __syncthreads();
                if (lane == 0) { sh.wave_rank[wave] = best; sh.wave_number[wave] = which; }
                __syncthreads();
                best = 0, which = ~0ull;
                for (int w = 0; w < kWaves; ++w)
                    if (sh.wave_rank[w] > best || (sh.wave_rank[w] == best && sh.wave_number[w] < which)) { best = sh.wave_rank[w]; which = sh.wave_number[w]; }
                if (best == 0) break;
                rank = __longlong_as_double(best >> 63 ? best & ~(1ull << 63) : ~best);
                number = which;
                if (tid == 0) write(found, rank, number);
            }
        }
        for (int i = found + tid; i < a.picks; i += kThreads) {
            a.out_parent[out + i] = a.out_token[out + i] = -1;
            a.out_score[out + i] = -INFINITY;
        }
    }
}

template <typename T, int PIECES> hipError_t beam(BeamArgs a, hipStream_t s)
{
    const int64_t groups = (int64_t)a.queries * a.beams * a.parts;
    k_beam_parts<T, PIECES><<<(unsigned)std::min<int64_t>(groups, 1 << 20), kThreads, 0, s>>>(a);
    if (hipError_t e = hipGetLastError()) return e;
    k_beam_queries<<<std::min(a.queries, 1 << 16), kThreads, 0, s>>>(a);
    return hipGetLastError();
}

template <typename T> int64_t parts_of(int32_t vocab) { return (vocab + Part<T, 8192 / kThreads / (16 / sizeof(T))>::SIZE - 1) / Part<T, 8192 / kThreads / (16 / sizeof(T))>::SIZE; }

}  // namespace

BeamSizes beam_sizes(int32_t queries, int32_t beams, int32_t vocab, int32_t picks, int32_t type)
{
    BeamSizes z{};
    z.parts = type == INFAAS_SEL_TYPE_FP32 ? parts_of<float>(vocab) : parts_of<bf16_t>(vocab);
    const int64_t groups = (int64_t)queries * beams * z.parts;
    z.sum_at = groups * picks * (int64_t)sizeof(u64);
    z.top_at = z.sum_at + groups * (int64_t)sizeof(double);
    z.bytes = z.top_at + groups * (int64_t)sizeof(float);
    return z;
}

hipError_t launch_beam(const BeamArgs &a, int32_t type, hipStream_t s)
{
    switch (type) {
    case INFAAS_SEL_TYPE_FP32: return beam<float, 8>(a, s);
    case INFAAS_SEL_TYPE_BF16: return beam<bf16_t, 4>(a, s);
    default: return beam<fp16_t, 4>(a, s);
    }
}

}  // namespace infaas
