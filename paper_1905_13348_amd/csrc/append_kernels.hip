// Appending keys and values to a paged cache with the rotation applied on the way (infaas_sel_exec_append).
#include "exec.h"

namespace infaas {

namespace {

template <typename T>
__device__ __forceinline__ vec<T, 8> load8(const void *p, int64_t at)
{
    return *(const vec<T, 8> *)((const T *)p + at);
}

template <typename T>
__device__ __forceinline__ void store8(void *p, int64_t at, vec<T, 8> v)
{
    *(vec<T, 8> *)((T *)p + at) = v;
}

// A workgroup takes one token; a thread takes the same sixteen dimensions of every so many heads, so that a sine and a
// cosine are computed once for all of them.  Rotated pairs lie in two vectors of eight: dimensions c*8.. and c*8 +
// rot/2.. (halves), or 16c.. (neighbours).
// What bounds it: memory from a few hundred tokens on (every element is read once and written once), below that the launch.
// 16,001 tokens of 32 + 8 + 8 heads of 128 in fp16, 393 MB: 89 us, 4.4 TB/s, where a large copy reaches 4.9; 1 and 128
// tokens: 7.2 us.
template <typename T>
__global__ __launch_bounds__(256) void k_append(AppendArgs p)
{
    const infaas_sel_append_args &a = p.a;
    const int D = p.head_dim, units = D / 16, half = a.rot_dim / 2;
    const int unit = threadIdx.x % units, lane = threadIdx.x / units, lanes = 256 / units;
    const int rot_units = a.rot_dim / 16;
    const int H = a.d_q ? p.heads : 0;
    for (int t = blockIdx.x; t < p.num_tokens; t += gridDim.x) {
        const int pos = p.token_pos[t], seq = p.token_seq[t];
        // where the key goes; -1: nowhere
        int64_t slot = -1;
        if (pos >= 0 && pos < p.cache.max_len && (uint32_t)seq < (uint32_t)p.num_seqs) {
            const int64_t page = p.cache.table[(int64_t)seq * p.cache.table_width + (pos >> p.cache.page_shift)];
            if (page >= 0 && page < p.cache.num_pages)
                slot = page * p.cache.page_stride + (int64_t)(pos & ((1 << p.cache.page_shift) - 1)) * p.cache.slot_stride;
        }
        const bool rotates = unit < rot_units;
        int d0 = unit * 16, d1 = d0 + 8;            // first dimensions of the two vectors
        float cs[8], sn[8];
        if (rotates) {
            if (!a.interleaved) { d0 = unit * 8; d1 = d0 + half; }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                // in turns: the fraction is what counts, and 32 bits are enough for that alone
                const double turns = (double)pos * a.d_freq[unit * 8 + i] * 0.15915494309189535;
                sincospif(2.0f * (float)(turns - rint(turns)), &sn[i], &cs[i]);
            }
        }
        for (int h = lane; h < H + 2 * p.kv_heads; h += lanes) {
            const bool is_q = h < H, is_k = !is_q && h < H + p.kv_heads;
            const int kvh = h - H - (is_k ? 0 : p.kv_heads);
            if (!is_q && slot < 0) continue;
            const void *src = is_q ? a.d_q : is_k ? a.d_k : a.d_v;
            const int64_t from = is_q ? t * a.q_token_stride + h * a.q_head_stride
                                 : is_k ? t * a.k_token_stride + kvh * a.k_head_stride
                                        : t * a.v_token_stride + kvh * a.v_head_stride;
            void *dst = is_q ? a.d_q_out : is_k ? p.cache.k : p.cache.v;
            const int64_t to = is_q ? t * a.out_token_stride + h * a.out_head_stride : slot + kvh * p.cache.head_stride;
            const int e0 = is_q || is_k ? d0 : unit * 16, e1 = is_q || is_k ? d1 : unit * 16 + 8;
            vec<T, 8> x = load8<T>(src, from + e0), y = load8<T>(src, from + e1);
            if (rotates && (is_q || is_k)) {
                if (a.interleaved) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float u = (float)x[2 * i], v = (float)x[2 * i + 1], w = (float)y[2 * i], z = (float)y[2 * i + 1];
                        x[2 * i] = (T)(u * cs[i] - v * sn[i]);
                        x[2 * i + 1] = (T)(v * cs[i] + u * sn[i]);
                        y[2 * i] = (T)(w * cs[4 + i] - z * sn[4 + i]);
                        y[2 * i + 1] = (T)(z * cs[4 + i] + w * sn[4 + i]);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float u = (float)x[i], v = (float)y[i];
                        x[i] = (T)(u * cs[i] - v * sn[i]);
                        y[i] = (T)(v * cs[i] + u * sn[i]);
                    }
                }
            }
            store8<T>(dst, to + e0, x);
            store8<T>(dst, to + e1, y);
        }
    }
}

}  // namespace

hipError_t launch_append(const AppendArgs &a, int32_t type, hipStream_t s)
{
    const dim3 grid(a.num_tokens < 65536 ? a.num_tokens : 65536);
    if (type == INFAAS_SEL_TYPE_BF16) k_append<bf16_t><<<grid, 256, 0, s>>>(a);
    else k_append<fp16_t><<<grid, 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace infaas
