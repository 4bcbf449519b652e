// Appending to a cache of 8 bits (infaas_sel_exec_append_scaled) and taking keys and values out of one (infaas_sel_exec_read).
#include "exec.h"

#include <algorithm>

namespace infaas {

namespace {

// ---- append -----------------------------------------------------------------------------------

// Sine and cosine of a position's turn, to 0.76 and 0.59 of a last place of 32 bits, 0.29 rms (half of one at most, and 0.29 rms, is the
// rounding itself).  In turns, of which quarters are taken off in 64 bits; what is left is an angle x of an eighth of a turn at most, as
// a number of 32 bits and what that leaves out.  sin x = x - x^3 / 6 + .., cos x = 1 - x^2 / 2 + ..: the leading terms are added with what
// their roundings leave out, the others (up to 0.08 and 0.02) in 32 bits; behind the last ones 1e-4 and 2e-3 of a place are left.
// (The series in 64 bits altogether: eleven registers more, and two waves to a SIMD instead of three.)
__device__ __forceinline__ float2 turned(int pos, double freq)
{
    const double turns = (double)pos * freq * 0.15915494309189535, q = rint(4 * turns), angle = (turns - 0.25 * q) * 6.283185307179586;
    const float x = (float)angle, rest = (float)(angle - (double)x), z = x * x;
    const float z_rest = __builtin_fmaf(x, x, -z) + 2 * x * rest;
    float p = 1.0f / 362880, c4 = -1.0f / 3628800;
    p = __builtin_fmaf(__builtin_fmaf(-1.0f / 39916800, z, p), z, -1.0f / 5040);
    p = __builtin_fmaf(__builtin_fmaf(p, z, 1.0f / 120), z, -1.0f / 6);
    c4 = __builtin_fmaf(__builtin_fmaf(c4, z, 1.0f / 40320), z, -1.0f / 720);
    c4 = __builtin_fmaf(c4, z, 1.0f / 24);
    const float s = x + __builtin_fmaf(x * z, p, rest * __builtin_fmaf(z, -0.5f, 1.0f));
    const float half = 0.5f * z, most = 1 - half;
    const float c = most + ((1 - most) - half + __builtin_fmaf(z * z, c4, -0.5f * z_rest));
    const int quarter = (int)(int64_t)q;
    const float sn = quarter & 1 ? c : s, cs = quarter & 1 ? s : c;
    return float2{quarter & 2 ? -sn : sn, (quarter + 1) & 2 ? -cs : cs};
}

// Sixteen dimensions of a head: two vectors of eight, d0.. and d1.., with eight rotated pairs or none.
struct Unit { int d0, d1; bool rotates; };
__device__ __forceinline__ Unit unit_of(const infaas_sel_append_args &a, int unit, bool rotated)
{
    const bool r = rotated && unit < a.rot_dim / 16;
    if (r && !a.interleaved) return Unit{unit * 8, unit * 8 + a.rot_dim / 2, true};
    return Unit{unit * 16, unit * 16 + 8, r};
}

template <typename T> struct Raw { vec<T, 8> a, b; };
template <typename T> __device__ __forceinline__ Raw<T> load16(const T *p, const Unit &u)
{
    return Raw<T>{*(const vec<T, 8> *)(p + u.d0), *(const vec<T, 8> *)(p + u.d1)};
}

// A unit's numbers, rotated by the eight sines and cosines at `turns` where it is.
template <typename T> __device__ __forceinline__ void numbers(const Raw<T> &r, const Unit &u, bool interleaved, const float2 *turns, float *x)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) { x[i] = (float)r.a[i]; x[8 + i] = (float)r.b[i]; }
    if (!u.rotates) return;
    float2 sc[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) sc[i] = turns[i];
    if (interleaved) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float p = x[2 * i], q = x[2 * i + 1];
            x[2 * i] = p * sc[i].y - q * sc[i].x;
            x[2 * i + 1] = q * sc[i].y + p * sc[i].x;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float p = x[i], q = x[8 + i];
            x[i] = p * sc[i].y - q * sc[i].x;
            x[8 + i] = q * sc[i].y + p * sc[i].x;
        }
    }
}

constexpr int kTurns = 4096;         // sines and cosines of a workgroup
constexpr int kHold = 8;             // rows that a thread holds

// The queries of some tokens.  Sines and cosines are computed once a token, and go through LDS.
template <typename T> __device__ __forceinline__ void append_queries(const AppendScaledArgs &p, int t0, float2 *turns)
{
    const infaas_sel_append_args &a = p.append.a;
    const int tid = threadIdx.x, half = a.rot_dim / 2, units = p.append.head_dim / 16, each = p.append.heads * units;
    const int tokens = min(p.q_tokens, p.append.num_tokens - t0), all = tokens * each;
    constexpr int DEEP = 4;      // units under way
    Raw<T> raw[DEEP];
    auto at = [&](int i, Unit &u, int &t, int &h) {
        t = i / each;
        const int r = i - t * each;
        h = r / units;
        u = unit_of(a, r - h * units, true);
        return r - h * units;
    };
    Unit u;
    int t, h;
    for (int i0 = 0; i0 < all; i0 += 256 * DEEP) {
#pragma unroll
        for (int d = 0; d < DEEP; ++d) {
            const int i = i0 + d * 256 + tid;
            if (i >= all) break;
            at(i, u, t, h);
            raw[d] = load16((const T *)a.d_q + (t0 + t) * a.q_token_stride + h * a.q_head_stride, u);
        }
        if (i0 == 0 && half) {
            for (int i = tid; i < tokens * half; i += 256) turns[i] = turned(p.append.token_pos[t0 + i / half], a.d_freq[i % half]);
            __syncthreads();
        }
#pragma unroll
        for (int d = 0; d < DEEP; ++d) {
            const int i = i0 + d * 256 + tid;
            if (i >= all) break;
            const int unit = at(i, u, t, h);
            float x[16];
            numbers(raw[d], u, a.interleaved, turns + t * half + unit * 8, x);
            T *to = (T *)a.d_q_out + (t0 + t) * a.out_token_stride + h * a.out_head_stride;
            vec<T, 8> y, z;
#pragma unroll
            for (int e = 0; e < 8; ++e) { y[e] = (T)x[e]; z[e] = (T)x[8 + e]; }
            *(vec<T, 8> *)(to + u.d0) = y;
            *(vec<T, 8> *)(to + u.d1) = z;
        }
    }
    __syncthreads();
}

// Keys and values of the blocks that begin with one of `chunk` tokens.  A column is the keys or the values of a KV head; a wave
// takes as many columns as leave each of its lanes `rows` tokens apart, a lane sixteen dimensions of up to eight rows, which stay in
// registers between the look at their largest and their rounding.  Nothing waits but for sines and cosines, which all heads share.
template <typename T> __device__ __forceinline__ void append_blocks(const AppendScaledArgs &p, int64_t chunk, int share, float2 *turns)
{
    const infaas_sel_append_args &a = p.append.a;
    const CacheArgs &c = p.append.cache;
    const int units = p.append.head_dim / 16, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int unit = lane % units, row = lane / units % p.rows, columns = 2 * p.append.kv_heads, side = 64 / (units * p.rows);
    const int64_t t0 = chunk * p.chunk;
    const int block = 1 << c.block_shift, page_mask = (1 << c.page_shift) - 1, half = a.rot_dim / 2;
    const int hold = p.rows * kHold;      // tokens of a wave at a time

    // The chunk's tokens with which a block begins for this step: the first of their block that is written (every wave looks at
    // all tokens of the chunk).
    bool first = false;
    int seq = 0, pos0 = 0, end = 0;
    const int64_t mine = t0 + lane;
    if (lane < p.chunk && mine < p.append.num_tokens) {
        seq = p.append.token_seq[mine];
        pos0 = p.append.token_pos[mine];
        if ((uint32_t)seq < (uint32_t)p.append.num_seqs) {
            const int s0 = p.seq_start[seq];
            end = min(p.seq_start[seq + 1], p.append.num_tokens);
            if (s0 >= 0 && mine >= s0 && mine < end) {
                const int64_t from = p.append.token_pos[s0];
                first = from >= 0 && pos0 == from + mine - s0;
                for (int64_t i = 1; first && i <= min(mine - s0, (int64_t)(pos0 & (block - 1))); ++i)
                    first = p.append.token_pos[mine - i] != pos0 - i || p.append.token_seq[mine - i] != seq;
            }
        }
    }
    unsigned long long leaders = __ballot(first);
    while (leaders) {
        const int l = __builtin_ctzll(leaders);
        leaders &= leaders - 1;
        const int64_t t = t0 + l;
        const int s = __builtin_amdgcn_readlane(seq, l), pos = __builtin_amdgcn_readlane(pos0, l);
        const int offset = pos & (block - 1), slot0 = (pos & page_mask) - offset;      // of the block's first key
        const int n = (int)min((int64_t)(block - offset), __builtin_amdgcn_readlane(end, l) - t);
        const int64_t page = page_of(c, s, p.append.num_seqs, pos);
        const bool many = n > hold;
        if (page < 0) continue;

        auto fill = [&](int i0) {      // sines and cosines of tokens i0 .. of the block
            if (many) __syncthreads();
            for (int i = tid; i < min(hold, n - i0) * half; i += 256) turns[i] = turned(pos + i0 + i / half, a.d_freq[i % half]);
            __syncthreads();
        };
        // the columns of this workgroup, `side` to a wave at a time
        for (int c0 = share * 4 * side; c0 < columns; c0 += p.shares * 4 * side) {
            const int column = c0 + wave * side + lane / (units * p.rows), head = min(column >> 1, p.append.kv_heads - 1);
            const bool keys = column % 2 == 0, here = column < columns;
            const Unit u = unit_of(a, unit, keys);
            const T *const src = keys ? (const T *)a.d_k + head * a.k_head_stride : (const T *)a.d_v + head * a.v_head_stride;
            const int64_t stride = keys ? a.k_token_stride : a.v_token_stride;
            uint8_t *const codes = (uint8_t *)(keys ? c.k : c.v) + head * c.head_stride + page * c.page_stride + (int64_t)slot0 * c.slot_stride;
            uint8_t *const scale = (keys ? c.k_scale : c.v_scale) + head * c.scale_head_stride + page * c.scale_page_stride +
                                   (int64_t)(slot0 >> c.block_shift) * c.scale_block_stride;
            const int old = *scale;
            Raw<T> raw[kHold];
            uint32_t held = 0;      // rows that are written
            auto load = [&](int i0) {
                held = 0;
#pragma unroll
                for (int r = 0; r < kHold; ++r) {
                    const int i = i0 + r * p.rows + row;
                    if (i0 + r * p.rows >= n) break;
                    if (i < n) {
                        raw[r] = load16(src + (t + i) * stride, u);
                        const bool there = pos + i < c.max_len && p.append.token_pos[t + i] == pos + i && p.append.token_seq[t + i] == s;
                        held |= (uint32_t)(there && here) << r;
                    }
                }
            };
            float top = 0;
            for (int i0 = 0; i0 < n; i0 += hold) {
                load(i0);
                if (half && (many || c0 == share * 4 * side)) fill(i0);
#pragma unroll
                for (int r = 0; r < kHold; ++r) {
                    if (i0 + r * p.rows >= n) break;
                    if (!(held >> r & 1)) continue;
                    float x[16];
                    numbers(raw[r], u, a.interleaved, turns + (r * p.rows + row) * half + unit * 8, x);
#pragma unroll
                    for (int e = 0; e < 16; ++e) top = fmaxf(top, fabsf(x[e]) < INFINITY ? fabsf(x[e]) : 0.0f);
                }
            }
            for (int d = 1; d < units * p.rows; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
            // the least e with top <= 1.75 * 2^(e - 127 + 8): the exponent, one more for a fraction beyond 1.75
            const int need = max(1, (int)((__float_as_uint(top) + 0x1fffff) >> 23) - 8);
            const int e = offset ? max(old, need) : need;
            if (offset && e > old && here) {      // (e > old: not of NaN)
                const float down = __uint_as_float((uint32_t)max(0, 127 + old - e) << 23);
                for (int i = row; i < offset; i += p.rows) {
                    vec<uint32_t, 4> *at = (vec<uint32_t, 4> *)(codes + i * c.slot_stride + unit * 16), w = *at;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w[j], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w[j], true);
                        w[j] = encode4(lo[0] * down, lo[1] * down, hi[0] * down, hi[1] * down);
                    }
                    *at = w;
                }
            }
            const float up = __uint_as_float(e < 254 ? (uint32_t)(254 - e) << 23 : 0x400000u);      // (2^-127 below the normal range)
            for (int i0 = 0; i0 < n; i0 += hold) {
                if (many) {
                    load(i0);
                    if (half) fill(i0);
                }
#pragma unroll
                for (int r = 0; r < kHold; ++r) {
                    if (i0 + r * p.rows >= n) break;
                    if (!(held >> r & 1)) continue;
                    float x[16];
                    numbers(raw[r], u, a.interleaved, turns + (r * p.rows + row) * half + unit * 8, x);
#pragma unroll
                    for (int j = 0; j < 16; ++j) x[j] *= up;
                    uint8_t *at = codes + (int64_t)(offset + i0 + r * p.rows + row) * c.slot_stride;
                    const vec<uint32_t, 2> lo = {encode4(x[0], x[1], x[2], x[3]), encode4(x[4], x[5], x[6], x[7])};
                    const vec<uint32_t, 2> hi = {encode4(x[8], x[9], x[10], x[11]), encode4(x[12], x[13], x[14], x[15])};
                    if (u.d1 == u.d0 + 8) {
                        *(vec<uint32_t, 4> *)(at + u.d0) = vec<uint32_t, 4>{lo[0], lo[1], hi[0], hi[1]};
                    } else {
                        *(vec<uint32_t, 2> *)(at + u.d0) = lo;
                        *(vec<uint32_t, 2> *)(at + u.d1) = hi;
                    }
                }
            }
            if (here && lane % (units * p.rows) == 0) *scale = (uint8_t)e;
        }
        if (half) __syncthreads();      // (before other sines and cosines come)
    }
}

// The workgroups in front take `chunk` tokens: of those they look for the ones with which a block begins for this step, and take
// these blocks one after the other.  The tokens of a block are known from the sequence's first one (their positions rise by
// one), so nothing is passed between workgroups and no order of atomics decides.  The others take the queries of some tokens each.
// What bounds it: 14,003 tokens of 32 + 8 + 8 heads of 128 in fp16, 316 MB, 83 us: 3.8 TB/s where a large copy reaches 5.2; vector
// instructions take half of the time (a code is computed twice, for its block's largest and for itself), and the 166 registers leave three
// waves to a SIMD to hide the trips to memory.  (With a workgroup to a block and head, and sines and cosines for each head, 167 us;
// queries in front 91.)  200 tokens, one to a sequence: 7 us, a launch and five trips to memory in a row.  A scale to every key
// makes a block of each token: 14,003 of them about 150 us.
template <typename T>
__global__ __launch_bounds__(256) void k_append_scaled(AppendScaledArgs p)
{
    __shared__ float2 turns[kTurns];
    const int blocks = gridDim.x - p.q_groups;
    if ((int)blockIdx.x >= blocks) {
        for (int64_t t = (int64_t)(blockIdx.x - blocks) * p.q_tokens; t < p.append.num_tokens; t += (int64_t)p.q_groups * p.q_tokens)
            append_queries<T>(p, (int)t, turns);
        return;
    }
    const int64_t all = ((int64_t)p.append.num_tokens + p.chunk - 1) / p.chunk * p.shares;
    for (int64_t g = blockIdx.x; g < all; g += blocks) append_blocks<T>(p, g / p.shares, (int)(g % p.shares), turns);
}

// ---- read -------------------------------------------------------------------------------------

// A thread takes sixteen dimensions of a token's key or value, of four tokens or parts of a token at a time: where they are is
// looked up for all four before their loads, since each look-up is three trips to memory in a row.  (19,000 tokens of 8 heads of
// 128 from codes, 117 MB: one part at a time 39 us, four 30, of sixteen dimensions instead of eight 27, 4.3 TB/s.)
template <typename T, bool CODED>
__global__ __launch_bounds__(256) void k_read(ReadArgs p)
{
    constexpr int DEEP = 4;
    const CacheArgs &c = p.cache;
    const uint32_t parts = p.head_dim / 16, each = 2 * p.kv_heads * parts;
    const int64_t all = (int64_t)each * p.num_tokens;
    for (int64_t i0 = (int64_t)blockIdx.x * 256 * DEEP; i0 < all; i0 += (int64_t)gridDim.x * 256 * DEEP) {
        const int64_t first = i0 / each;                                // (the same for the workgroup)
        const uint32_t rest = (uint32_t)(i0 - first * each) + threadIdx.x;
        int64_t token[DEEP], page[DEEP];
        uint32_t part[DEEP];
        int pos[DEEP], seq[DEEP];
#pragma unroll
        for (int d = 0; d < DEEP; ++d) {
            const uint32_t r = rest + d * 256;
            token[d] = first + r / each;
            part[d] = r % each;
            const int64_t t = min(token[d], (int64_t)p.num_tokens - 1);
            pos[d] = p.token_pos[t];
            seq[d] = p.token_seq[t];
        }
#pragma unroll
        for (int d = 0; d < DEEP; ++d) page[d] = page_of(c, seq[d], p.num_seqs, pos[d]);
        vec<uint32_t, 4> raw[DEEP][2];
        uint32_t e[DEEP];
#pragma unroll
        for (int d = 0; d < DEEP; ++d) {
            const bool keys = part[d] < p.kv_heads * parts;
            const int head = (int)(part[d] / parts % p.kv_heads), slot = pos[d] & ((1 << c.page_shift) - 1);
            const int64_t there = max(page[d], (int64_t)0);
            const int64_t at = page[d] < 0 ? 0 : there * c.page_stride + slot * c.slot_stride + head * c.head_stride + part[d] % parts * 16;
            const void *pool = keys ? c.k : c.v;
            if (CODED) {
                e[d] = (keys ? c.k_scale : c.v_scale)[page[d] < 0 ? 0 : there * c.scale_page_stride +
                                                                          (slot >> c.block_shift) * c.scale_block_stride + head * c.scale_head_stride];
                raw[d][0] = *(const vec<uint32_t, 4> *)((const uint8_t *)pool + at);
            } else {
                raw[d][0] = *(const vec<uint32_t, 4> *)((const T *)pool + at);
                raw[d][1] = *(const vec<uint32_t, 4> *)((const T *)pool + at + 8);
            }
        }
#pragma unroll
        for (int d = 0; d < DEEP; ++d) {
            if (token[d] >= p.num_tokens) continue;
            const bool keys = part[d] < p.kv_heads * parts;
            const int head = (int)(part[d] / parts % p.kv_heads);
            T *to = keys ? (T *)p.k + token[d] * p.k_token_stride + head * p.k_head_stride : (T *)p.v + token[d] * p.v_token_stride + head * p.v_head_stride;
            to += part[d] % parts * 16;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                union { vec<T, 8> v; vec<uint32_t, 4> w; } u;
                if (CODED) u.v = decode8<T>(vec<uint32_t, 2>{raw[d][0][2 * h], raw[d][0][2 * h + 1]}, e[d]);
                else u.w = raw[d][h];
                if (page[d] < 0) u.w = vec<uint32_t, 4>{};
                *(vec<uint32_t, 4> *)(to + 8 * h) = u.w;
            }
        }
    }
}

template <typename T>
hipError_t read(const ReadArgs &a, hipStream_t s)
{
    const int64_t all = (int64_t)2 * a.kv_heads * (a.head_dim / 16) * a.num_tokens;
    const dim3 grid((unsigned)std::min<int64_t>(kMostGroups, (all + 1023) / 1024));
    if (a.cache.k_scale) k_read<T, true><<<grid, 256, 0, s>>>(a);
    else k_read<T, false><<<grid, 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_append_scaled(const AppendScaledArgs &args, int32_t type, hipStream_t s)
{
    AppendScaledArgs a = args;
    const int64_t n = a.append.num_tokens, block = 1ll << a.append.cache.block_shift;
    const int units = a.append.head_dim / 16, columns = 2 * a.append.kv_heads;
    // Queries: as many tokens to a workgroup as there are sines and cosines of, at most four, one where there are few.
    a.q_tokens = (int)std::max<int64_t>(1, std::min<int64_t>(4, n / 512));
    a.q_groups = a.append.a.d_q ? (int)std::min<int64_t>((n + a.q_tokens - 1) / a.q_tokens, kMostGroups) : 0;
    // Rows side by side: a power of two up to the tokens of a block (on an average, sequences are as long as each other), so that
    // with single tokens a wave has several columns.
    const int64_t run = std::max<int64_t>(1, std::min<int64_t>(block, n / std::max(1, a.append.num_seqs)));
    a.rows = 1;
    while (2 * a.rows <= run && 2 * a.rows * units <= 64) a.rows *= 2;
    // A chunk to a workgroup is a block's tokens at most (64 at most: a wave looks them through), one where there are few; columns
    // are shared among workgroups until there are 2048 of these.
    a.chunk = (int)std::max<int64_t>(1, std::min<int64_t>({64, block, n / 512}));
    const int64_t chunks = (n + a.chunk - 1) / a.chunk;
    const int at_once = 4 * (64 / (units * a.rows));
    const int64_t most = (columns + at_once - 1) / at_once;
    a.shares = (int)std::max<int64_t>(1, std::min<int64_t>(most, 2048 / std::max<int64_t>(1, chunks) + 1));
    const int64_t groups = std::min<int64_t>(chunks * a.shares, kMostGroups);
    const dim3 grid((unsigned)(groups + a.q_groups));
    if (type == INFAAS_SEL_TYPE_BF16) k_append_scaled<bf16_t><<<grid, 256, 0, s>>>(a);
    else k_append_scaled<fp16_t><<<grid, 256, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_read(const ReadArgs &a, int32_t type, hipStream_t s)
{
    return type == INFAAS_SEL_TYPE_BF16 ? read<bf16_t>(a, s) : read<fp16_t>(a, s);
}

}  // namespace infaas
