// Drawing a token of every row of logits (infaas_sel_exec_sample).
#include "exec.h"

namespace infaas {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kSegments = 2048;              // stretches of a row whose sums are kept for the draw
constexpr int kShift = 43;                   // a weight of 1 is 2^43: 2^20 of them stay below 2^63
constexpr uint32_t kNever = 0x007fffffu;     // order key of -infinity

typedef unsigned long long u64;

// Logits as 32-bit numbers in their order: equal logits (-0 and +0, too) have equal keys; NaN counts as -infinity.
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t b = __float_as_uint(x + 0.0f);
    const uint32_t k = b >> 31 ? ~b : b | 0x80000000u;
    return x != x ? kNever : k;
}
__device__ __forceinline__ float value_of(uint32_t k) { return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k); }

template <typename T> __device__ __forceinline__ uint32_t load_key(const T *row, int i) { return key_of((float)row[i]); }

// exp((x - top) / temperature) in 64 bits; among +infinities 1.
struct Weights {
    double top, per_t;
    bool infinite;
    __device__ __forceinline__ double real(uint32_t k) const
    {
        if (k <= kNever) return 0.0;
        const float x = value_of(k);
        if (infinite) return x == INFINITY ? 1.0 : 0.0;
        const double y = ((double)x - top) * per_t;
        return y < -40.0 ? 0.0 : exp(y);
    }
    __device__ __forceinline__ u64 fixed(double w) const { return (u64)rint(w * (double)(1ull << kShift)); }
    __device__ __forceinline__ u64 operator()(uint32_t k) const { return fixed(real(k)); }
};

// What is kept: everything above `key`, and of the tokens at `key` those numbered up to `last`.
struct Kept {
    uint32_t key;
    int last;
    __device__ __forceinline__ bool has(uint32_t k, int i) const { return k > key || (k == key && i <= last); }
};

struct Shared {
    u64 mass[256];
    uint32_t count[256];
    u64 seg[kSegments];
    u64 wave_sum[kWaves];
    uint32_t key;
    u64 left;
    int index;
    u64 total;
};

__device__ __forceinline__ u64 wave_sum(u64 v)
{
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// Running sums over sh.seg[0 .. n-1] in place (each entry: what is in front of it); returns the total.  All threads.
__device__ u64 scan_segments(Shared &sh, int n)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    constexpr int EACH = kSegments / kThreads;
    u64 v[EACH], sum = 0;
    for (int e = 0; e < EACH; ++e) {
        const int i = tid * EACH + e;
        v[e] = i < n ? sh.seg[i] : 0;
        sum += v[e];
    }
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
    for (int e = 0; e < EACH; ++e) {
        const int i = tid * EACH + e;
        if (i < n) sh.seg[i] = before;
        before += v[e];
    }
    __syncthreads();
    return all;
}

// The token, in the order of numbers, whose measure f(i), added to what is in front of it, first exceeds `at`
// (at < the sum of all).  sh.seg holds the running sums of the segments.  All threads get the answer.
template <typename F> __device__ int find_in_order(Shared &sh, int V, int seg_len, int segs, u64 at, F f)
{
    const int tid = threadIdx.x, lane = tid & 63;
    for (int i = tid; i < segs; i += kThreads) {
        const u64 next = i + 1 < segs ? sh.seg[i + 1] : ~0ull;
        if (sh.seg[i] <= at && at < next) sh.index = i;      // (of segments that add nothing the last: one thread)
    }
    __syncthreads();
    const int seg = sh.index;
    __syncthreads();
    if (tid < 64) {
        u64 before = sh.seg[seg];
        const int end = min(V, (seg + 1) * seg_len);
        int found = -1;
        for (int i0 = seg * seg_len; i0 < end && found < 0; i0 += 64) {
            const int i = i0 + lane;
            const u64 w = i < end ? f(i) : 0;
            u64 inc = w;
            for (int d = 1; d < 64; d <<= 1) {
                const u64 o = __shfl_up(inc, d);
                if (lane >= d) inc += o;
            }
            const u64 hit = __ballot(w > 0 && before + inc > at);
            if (hit) found = i0 + __ffsll(hit) - 1;
            before += __shfl(inc, 63);
        }
        if (lane == 0) sh.index = found;
    }
    __syncthreads();
    return sh.index;
}

// Of the tokens in `within`, from the greatest: the one at which the number of tokens (by_mass: the sum of their
// weights) reaches `target` >= 1, as the border of what is then kept.  If it is never reached, everything is.
template <typename T, bool by_mass>
__device__ Kept select(Shared &sh, const T *row, int V, int seg_len, int segs, const Weights &wt, Kept within, u64 target)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    uint32_t prefix = 0;
    u64 left = target, ties = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = tid; i < 256; i += kThreads) sh.count[i] = 0, sh.mass[i] = 0;
        __syncthreads();
        const uint32_t mask = shift == 24 ? 0u : ~0u << (shift + 8);
        for (int i = tid; i < V; i += kThreads) {
            const uint32_t k = load_key(row, i);
            if ((k & mask) == prefix && k > kNever && within.has(k, i)) {
                atomicAdd(&sh.count[k >> shift & 255], 1u);
                if (by_mass) atomicAdd(&sh.mass[k >> shift & 255], wt(k));
            }
        }
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
    // of the tokens with this key the first so many
    u64 m = by_mass ? (left + wt(prefix) - 1) / wt(prefix) : left;
    if (m >= ties) return Kept{prefix, prefix == within.key ? within.last : 0x7fffffff};
    for (int s = wave; s < segs; s += kWaves) {
        u64 c = 0;
        for (int i = s * seg_len + lane; i < min(V, (s + 1) * seg_len); i += 64) c += load_key(row, i) == prefix;
        c = wave_sum(c);
        if (lane == 0) sh.seg[s] = c;
    }
    __syncthreads();
    scan_segments(sh, segs);
    const int last = find_in_order(sh, V, seg_len, segs, m - 1, [&](int i) -> u64 { return load_key(row, i) == prefix; });
    return Kept{prefix, last};
}

// A workgroup per row.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_sample(SampleArgs a)
{
    __shared__ Shared sh;
    const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, V = a.vocab;
    const T *row = (const T *)a.logits + r * a.row_stride;
    const int seg_len = 64 * ((V + 64 * kSegments - 1) / (64 * kSegments)), segs = (V + seg_len - 1) / seg_len;

    if (tid == 0) sh.key = 0;
    __syncthreads();
    uint32_t top = 0;
    for (int i = tid; i < V; i += kThreads) top = max(top, load_key(row, i));
    for (int d = 32; d; d >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
    if (lane == 0) atomicMax(&sh.key, top);
    __syncthreads();
    top = sh.key;
    __syncthreads();

    if (top <= kNever) {
        if (tid == 0) {
            a.token[r] = -1;
            if (a.prob) a.prob[r] = 0.0f;
        }
        return;
    }
    const float t = a.temperature ? a.temperature[r] : 1.0f;
    const float top_p = a.top_p ? a.top_p[r] : 1.0f, min_p = a.min_p && a.min_p[r] > 0 ? a.min_p[r] : 0.0f;
    const bool first = !(t > 0) || min_p > 1.0f;
    const int k = first ? 1 : a.top_k ? a.top_k[r] : 0;
    Weights wt;
    wt.top = value_of(top);
    wt.infinite = value_of(top) == INFINITY;
    wt.per_t = first ? 1.0 : 1.0 / (double)t;

    Kept kept{kNever, 0x7fffffff};
    if (k > 0 && k < V) kept = select<T, false>(sh, row, V, seg_len, segs, wt, kept, (u64)k);
    auto sums = [&](double least) {      // of what is kept, in segments
        for (int s = wave; s < segs; s += kWaves) {
            u64 c = 0;
            for (int i = s * seg_len + lane; i < min(V, (s + 1) * seg_len); i += 64) {
                const uint32_t x = load_key(row, i);
                if (kept.has(x, i)) {
                    const double w = wt.real(x);
                    if (w >= least) c += wt.fixed(w);
                }
            }
            c = wave_sum(c);
            if (lane == 0) sh.seg[s] = c;
        }
        __syncthreads();
        return scan_segments(sh, segs);
    };
    if (!first && top_p < 1.0f) {
        const u64 total = sums(0.0);
        const double need = ceil((double)top_p * (double)total);
        kept = select<T, true>(sh, row, V, seg_len, segs, wt, kept, need >= 1.0 ? (u64)need : 1ull);
    }
    const double least = first ? 0.0 : (double)min_p;
    const u64 total = sums(least);
    const double at = floor((double)(a.draw[r]) * (double)total);
    const u64 pick = at > 0 ? min((u64)at, total - 1) : 0;
    const int token = find_in_order(sh, V, seg_len, segs, pick, [&](int i) -> u64 {
        const uint32_t x = load_key(row, i);
        if (!kept.has(x, i)) return 0;
        const double w = wt.real(x);
        return w >= least ? wt.fixed(w) : 0;
    });
    if (tid == 0) {
        a.token[r] = token;
        if (a.prob) a.prob[r] = (float)((double)wt(load_key(row, token)) / (double)total);
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
