// Appending to a cache of 8 bits (infaas_sel_exec_append_scaled) and taking keys and values out of one (infaas_sel_exec_read).
#include "exec.h"

#include <algorithm>

namespace infaas {

namespace {

// ---- append -----------------------------------------------------------------------------------

// Sine and cosine of eight neighbouring rotated pairs.
__device__ __forceinline__ void angles(const double *freq, int pos, float *sn, float *cs)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        // In turns, of which quarters are taken off in 64 bits: what is left is an eighth at most, and keeps its bits in 32.  (With
        // whole turns taken off alone an angle near a half or a whole one is off by 2e-7: five times as many codes fall on the
        // other side of a border.)
        const double turns = (double)pos * freq[i] * 0.15915494309189535, q = rint(4 * turns);
        float s, c;
        sincospif(2.0f * (float)(turns - 0.25 * q), &s, &c);
        const int quarter = (int)(int64_t)q;
        sn[i] = quarter & 1 ? c : s;
        cs[i] = quarter & 1 ? s : c;
        sn[i] = quarter & 2 ? -sn[i] : sn[i];
        cs[i] = (quarter + 1) & 2 ? -cs[i] : cs[i];
    }
}

// Sixteen dimensions of a head: two vectors of eight, d0.. and d1.., with eight rotated pairs or none.
struct Unit { int d0, d1; bool rotates; };
__device__ __forceinline__ Unit unit_of(const infaas_sel_append_args &a, int unit, bool rotated)
{
    const bool r = rotated && unit < a.rot_dim / 16;
    if (r && !a.interleaved) return Unit{unit * 8, unit * 8 + a.rot_dim / 2, true};
    return Unit{unit * 16, unit * 16 + 8, r};
}

template <typename T> __device__ __forceinline__ void load16(const T *p, const Unit &u, float *x)
{
    const vec<T, 8> a = *(const vec<T, 8> *)(p + u.d0), b = *(const vec<T, 8> *)(p + u.d1);
#pragma unroll
    for (int i = 0; i < 8; ++i) { x[i] = (float)a[i]; x[8 + i] = (float)b[i]; }
}

__device__ __forceinline__ void rotate16(float *x, bool interleaved, const float *sn, const float *cs)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float &p = x[interleaved ? 2 * i : i], &q = x[interleaved ? 2 * i + 1 : 8 + i];
        const float u = p, v = q;
        p = u * cs[i] - v * sn[i];
        q = v * cs[i] + u * sn[i];
    }
}

// A KV head's keys or its values, of the blocks that begin with one of `chunk` tokens.
template <typename T> __device__ __forceinline__ void append_blocks(const AppendScaledArgs &p, int64_t g, float *tops)
{
    const infaas_sel_append_args &a = p.append.a;
    const CacheArgs &c = p.append.cache;
    const int units = p.append.head_dim / 16, tid = threadIdx.x, unit = tid % units, lane = tid / units, lanes = 256 / units;
    const int head = (int)(g / 2 % p.append.kv_heads);
    const bool keys = g % 2 == 0;
    const int64_t t0 = g / 2 / p.append.kv_heads * p.chunk;
    const T *const src = keys ? (const T *)a.d_k + head * a.k_head_stride : (const T *)a.d_v + head * a.v_head_stride;
    const int64_t stride = keys ? a.k_token_stride : a.v_token_stride;
    uint8_t *const pool = (uint8_t *)(keys ? c.k : c.v) + head * c.head_stride;
    uint8_t *const scales = (keys ? c.k_scale : c.v_scale) + head * c.scale_head_stride;
    const Unit u = unit_of(a, unit, keys);
    const int block = 1 << c.block_shift, page_mask = (1 << c.page_shift) - 1;

    // The chunk's tokens with which a block begins for this step: the first of their block that is written (every wave looks at
    // all tokens of the chunk).
    bool first = false;
    const int64_t mine = t0 + (tid & 63);
    if ((tid & 63) < p.chunk && mine < p.append.num_tokens) {
        const int s = p.append.token_seq[mine];
        if ((uint32_t)s < (uint32_t)p.append.num_seqs) {
            const int s0 = p.seq_start[s], s1 = min(p.seq_start[s + 1], p.append.num_tokens);
            if (s0 >= 0 && mine >= s0 && mine < s1) {
                const int64_t from = p.append.token_pos[s0], pos = from + mine - s0;
                first = from >= 0 && p.append.token_pos[mine] == pos;
                for (int64_t i = 1; first && i <= min(mine - s0, pos & (block - 1)); ++i)
                    first = p.append.token_pos[mine - i] != pos - i || p.append.token_seq[mine - i] != s;
            }
        }
    }
    unsigned long long leaders = __ballot(first);
    while (leaders) {
        const int64_t t = t0 + __builtin_ctzll(leaders);
        leaders &= leaders - 1;
        const int s = p.append.token_seq[t], pos = p.append.token_pos[t];
        const int64_t page = page_of(c, s, p.append.num_seqs, pos);
        if (page < 0) continue;
        const int offset = pos & (block - 1), slot0 = (pos & page_mask) - offset;      // of the block's first key
        const int n = (int)min((int64_t)(block - offset), min(p.seq_start[s + 1], p.append.num_tokens) - t);
        uint8_t *const codes = pool + page * c.page_stride + (int64_t)slot0 * c.slot_stride;
        uint8_t *const scale = scales + page * c.scale_page_stride + (slot0 >> c.block_shift) * c.scale_block_stride;
        auto there = [&](int i) {
            return pos + i < c.max_len && p.append.token_pos[t + i] == pos + i && p.append.token_seq[t + i] == s;
        };
        auto number = [&](int i, float *x) {
            load16(src + (t + i) * stride, u, x);
            if (u.rotates) {
                float sn[8], cs[8];
                angles(a.d_freq + unit * 8, pos + i, sn, cs);
                rotate16(x, a.interleaved, sn, cs);
            }
        };
        float top = 0;
        for (int i = lane; i < n; i += lanes) {
            float x[16];
            if (!there(i)) continue;
            number(i, x);
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, fabsf(x[e]) < INFINITY ? fabsf(x[e]) : 0.0f);
        }
        for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
        __syncthreads();
        if ((tid & 63) == 0) tops[tid >> 6] = top;
        const int old = *scale;
        __syncthreads();
        top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
        // the least e with top <= 1.75 * 2^(e - 127 + 8): the exponent, one more for a fraction beyond 1.75
        const int need = max(1, (int)((__float_as_uint(top) + 0x1fffff) >> 23) - 8);
        const int e = offset ? max(old, need) : need;
        if (offset && e > old) {      // (e > old: not of NaN)
            const float down = __uint_as_float((uint32_t)max(0, 127 + old - e) << 23);
            for (int i = lane; i < offset; i += lanes) {
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
        for (int i = lane; i < n; i += lanes) {
            float x[16];
            if (!there(i)) continue;
            number(i, x);
#pragma unroll
            for (int j = 0; j < 16; ++j) x[j] *= up;
            uint8_t *at = codes + (offset + i) * c.slot_stride;
            *(vec<uint32_t, 2> *)(at + u.d0) = vec<uint32_t, 2>{encode4(x[0], x[1], x[2], x[3]), encode4(x[4], x[5], x[6], x[7])};
            *(vec<uint32_t, 2> *)(at + u.d1) = vec<uint32_t, 2>{encode4(x[8], x[9], x[10], x[11]), encode4(x[12], x[13], x[14], x[15])};
        }
        __syncthreads();
        if (tid == 0) *scale = (uint8_t)e;
    }
}

// The workgroups in front rotate the queries, a token each.  The others take a KV head's keys or its values, and `chunk`
// tokens: of those they look for the ones with which a block begins for this step, and take these blocks one after the other.
// The tokens of a block are known from the sequence's first one (their positions rise by one), so nothing is passed between
// workgroups and no order of atomics decides.
template <typename T>
__global__ __launch_bounds__(256) void k_append_scaled(AppendScaledArgs p)
{
    const infaas_sel_append_args &a = p.append.a;
    const CacheArgs &c = p.append.cache;
    const int D = p.append.head_dim, units = D / 16, tid = threadIdx.x;
    const int unit = tid % units, lane = tid / units, lanes = 256 / units;
    if ((int)blockIdx.x < p.q_groups) {
        const Unit u = unit_of(a, unit, true);
        for (int t = blockIdx.x; t < p.append.num_tokens; t += p.q_groups) {
            float sn[8], cs[8], x[16];
            if (u.rotates) angles(a.d_freq + unit * 8, p.append.token_pos[t], sn, cs);
            for (int h = lane; h < p.append.heads; h += lanes) {
                load16((const T *)a.d_q + t * a.q_token_stride + h * a.q_head_stride, u, x);
                if (u.rotates) rotate16(x, a.interleaved, sn, cs);
                T *to = (T *)a.d_q_out + t * a.out_token_stride + h * a.out_head_stride;
                vec<T, 8> y, z;
#pragma unroll
                for (int i = 0; i < 8; ++i) { y[i] = (T)x[i]; z[i] = (T)x[8 + i]; }
                *(vec<T, 8> *)(to + u.d0) = y;
                *(vec<T, 8> *)(to + u.d1) = z;
            }
        }
        return;
    }
    __shared__ float tops[4];
    const int64_t chunks = ((int64_t)p.append.num_tokens + p.chunk - 1) / p.chunk;
    for (int64_t g = blockIdx.x - p.q_groups; g < chunks * 2 * p.append.kv_heads; g += gridDim.x - p.q_groups) append_blocks<T>(p, g, tops);
}

// ---- read -------------------------------------------------------------------------------------

// A thread takes sixteen bytes of the result: eight dimensions of a token's key or value.
template <typename T, bool CODED>
__global__ __launch_bounds__(256) void k_read(ReadArgs p)
{
    const int parts = p.head_dim / 8;
    const int64_t each = (int64_t)2 * p.kv_heads * parts, all = each * p.num_tokens;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const int64_t t = i / each;
        const int r = (int)(i - t * each), head = r / parts % p.kv_heads, d = r % parts * 8;
        const bool keys = r < p.kv_heads * parts;
        const CacheArgs &c = p.cache;
        const int pos = p.token_pos[t];
        const int64_t page = page_of(c, p.token_seq[t], p.num_seqs, pos);
        vec<T, 8> y = vec<T, 8>{};
        if (page >= 0) {
            const int slot = pos & ((1 << c.page_shift) - 1);
            const int64_t at = page * c.page_stride + slot * c.slot_stride + head * c.head_stride + d;
            if (CODED) {
                const uint32_t e = (keys ? c.k_scale : c.v_scale)[page * c.scale_page_stride +
                                                                  (slot >> c.block_shift) * c.scale_block_stride + head * c.scale_head_stride];
                y = decode8<T>(*(const vec<uint32_t, 2> *)((const uint8_t *)(keys ? c.k : c.v) + at), e);
            } else {
                y = *(const vec<T, 8> *)((const T *)(keys ? c.k : c.v) + at);
            }
        }
        T *to = keys ? (T *)p.k + t * p.k_token_stride + head * p.k_head_stride : (T *)p.v + t * p.v_token_stride + head * p.v_head_stride;
        *(vec<T, 8> *)(to + d) = y;
    }
}

template <typename T>
hipError_t read(const ReadArgs &a, hipStream_t s)
{
    const int64_t all = (int64_t)2 * a.kv_heads * (a.head_dim / 8) * a.num_tokens;
    const dim3 grid((unsigned)std::min<int64_t>(kMostGroups, (all + 255) / 256));
    if (a.cache.k_scale) k_read<T, true><<<grid, 256, 0, s>>>(a);
    else k_read<T, false><<<grid, 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_append_scaled(const AppendScaledArgs &args, int32_t type, hipStream_t s)
{
    AppendScaledArgs a = args;
    const int64_t n = a.append.num_tokens, block = 1ll << a.append.cache.block_shift, pairs = 2ll * a.append.kv_heads;
    a.q_groups = a.append.a.d_q ? (int)std::min<int64_t>(n, kMostGroups) : 0;
    // A chunk to a workgroup is a block's tokens at most (64 at most: a wave looks them through), one where there are few.
    a.chunk = (int)std::max<int64_t>(1, std::min<int64_t>({64, block, n / 512}));
    const int64_t groups = std::min<int64_t>((n + a.chunk - 1) / a.chunk * pairs, kMostGroups);
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
