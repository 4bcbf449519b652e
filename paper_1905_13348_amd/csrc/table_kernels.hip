// The pages of a worker's sequences (infaas_sel_exec_advance) and copies of pages (infaas_sel_exec_copy).
#include "exec.h"

#include <algorithm>

namespace infaas {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
typedef long long i64;

__device__ __forceinline__ int pages_of(const AdvanceArgs &a, int keys) { return (int)(((i64)keys + a.t.page_size - 1) >> a.page_shift); }
__device__ __forceinline__ int length_of(const AdvanceArgs &a, int s) { return min(max(a.t.d_seq_len[s], 0), a.most); }
__device__ __forceinline__ bool is_page(const AdvanceArgs &a, int page) { return (uint32_t)page < (uint32_t)a.t.num_pages; }
// The sequence whose state a sequence goes on from, or -1.
__device__ __forceinline__ int parent_of(const AdvanceArgs &a, int s)
{
    if (!a.parent) return s;
    const int p = a.parent[s];
    return (uint32_t)p < (uint32_t)a.t.num_seqs ? p : -1;
}

// ---- rows that go on from others ----------------------------------------------------------------

// A workgroup takes some columns of the table, of all rows: what the rows are to be is read before any is written.  Counts
// change by atomics, whose order does not matter.  (4 us: a launch and four trips to memory in a row.)
constexpr int kCells = 8192;
__global__ __launch_bounds__(kThreads) void k_reparent(AdvanceArgs a, int columns)
{
    __shared__ int cell[kCells];
    const int S = a.t.num_seqs;
    for (i64 c0 = (i64)blockIdx.x * columns; c0 < a.t.table_width; c0 += (i64)gridDim.x * columns) {
        for (int i = threadIdx.x; i < S * columns; i += kThreads) {
            const int s = i / columns, p = parent_of(a, s);
            const i64 c = c0 + i % columns;
            cell[i] = p >= 0 && p != s && c < pages_of(a, length_of(a, p)) ? a.t.d_page_table[(i64)p * a.t.table_width + c] : -1;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < S * columns; i += kThreads) {
            const int s = i / columns, p = parent_of(a, s);
            const i64 c = c0 + i % columns;
            if (p == s) continue;
            const int had = pages_of(a, length_of(a, s)), has = p < 0 ? 0 : pages_of(a, length_of(a, p));
            if (c >= max(had, has)) continue;
            int32_t *const at = a.t.d_page_table + (i64)s * a.t.table_width + c;
            const int before = c < had ? *at : -1, now = cell[i];
            *at = now;
            if (before == now) continue;
            if (is_page(a, before)) atomicSub(&a.t.d_page_refs[before], 1);
            if (is_page(a, now)) atomicAdd(&a.t.d_page_refs[now], 1);
        }
        __syncthreads();
    }
}

// ---- lengths, pages, the batch's arrays ---------------------------------------------------------

// What is in front of a thread, and the sum over all threads, both saturating at 2^32 - 1: more of anything than there is of it
// in any case.
struct InFront { uint32_t before, all; };
__device__ __forceinline__ uint32_t plus(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }

// Running sums over a wave, each lane's own included: within rows of 16 lanes, then the last lane of a row into the next, and of
// the lower half into the upper.
__device__ __forceinline__ uint32_t upto_me(uint32_t x)
{
    x = plus(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false));
    x = plus(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, false));
    x = plus(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, false));
    x = plus(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, false));
    x = plus(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false));
    return plus(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false));
}

// Of N values at once.  (Two barriers.)
template <int N> __device__ __forceinline__ void in_front(const uint32_t (&v)[N], uint32_t (*waves)[kWaves], InFront (&out)[N])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t inc[N];
#pragma unroll
    for (int i = 0; i < N; ++i) inc[i] = upto_me(v[i]);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (lane == 63) waves[i][wave] = inc[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        // (the waves' sums in the lanes of a row)
        const uint32_t sums = upto_me(lane < kWaves ? waves[i][lane] : 0);
        out[i].all = (uint32_t)__builtin_amdgcn_readlane((int)sums, kWaves - 1);
        const uint32_t others = wave ? (uint32_t)__builtin_amdgcn_readlane((int)sums, wave - 1) : 0;
        const uint32_t mine = (uint32_t)__shfl_up((int)inc[i], 1);
        out[i].before = plus(others, lane ? mine : 0);
    }
}

// The last of n entries, which do not fall, that is at most x (the first is).
__device__ __forceinline__ int last_upto(const int *v, int n, int x)
{
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (v[mid] <= x) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// Sequence and position of tokens first, first + step, ...; `start` are the sequences' first tokens, `shift` what makes of a
// token's number its position.
__device__ __forceinline__ void fill_tokens(const AdvanceArgs &a, const int *start, const int *shift, int total, int first, int step)
{
    for (i64 i = first; i < a.t.max_tokens; i += step) {
        int seq = -1, pos = -1;
        if (i < total) {
            seq = last_upto(start, a.t.num_seqs, (int)i);
            pos = shift[seq] + (int)i;
        }
        a.t.d_token_seq[i] = seq;
        a.t.d_token_pos[i] = pos;
    }
}

// Batches of more tokens are written by a launch of their own.
constexpr int kFewTokens = 4096;

// One workgroup; thread t has sequences t, t + 1024, ...  What bounds it is the chain of its steps, each a trip to memory or a
// barrier, and the first fetch of its instructions: so few sequences have a shorter code, sums are taken two at a time and only
// where they may differ from what is known, and the counts of pages are under way from the start.  (256 sequences that drop drafts or
// take some 8 to 10 us, before that 17; 300 prompts 10.4, before that 20; 4096 sequences, four to a thread, 33.)
template <int ROWS>
__global__ __launch_bounds__(kThreads) void k_advance(AdvanceArgs a)
{
    __shared__ int base[ROWS * kThreads];      // pages that those in front of a sequence need; at the end its first token
    __shared__ int column[ROWS * kThreads];    // where its first new page goes; as ~column, where that is for a copy; at the end its shift
    __shared__ uint32_t waves[2][kWaves];
    const int S = a.t.num_seqs, W = a.t.table_width, P = a.t.page_size, tid = threadIdx.x, lane = tid & 63;
    int32_t *const refs = a.t.d_page_refs;
    constexpr int EACH = 16;      // pages of a thread at a time
    int4 counts[EACH / 4];
    auto load_counts = [&](i64 p0) {
        const i64 mine = p0 + tid * EACH;
#pragma unroll
        for (int q = 0; q < EACH / 4; ++q)
            if (mine + 4 * q + 4 <= a.t.num_pages) counts[q] = *(const int4 *)(refs + mine + 4 * q);
            else counts[q] = int4{mine + 4 * q < a.t.num_pages ? refs[mine + 4 * q] : 1, mine + 4 * q + 1 < a.t.num_pages ? refs[mine + 4 * q + 1] : 1,
                                  mine + 4 * q + 2 < a.t.num_pages ? refs[mine + 4 * q + 2] : 1, 1};
    };
    load_counts(0);

    // what goes
    int len[ROWS], more[ROWS], need[ROWS], last[ROWS];      // last: the page to copy, or -1
    bool gave = false;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const int s = r * kThreads + tid;
        len[r] = more[r] = 0;
        int had = 0, has = 0;
        if (s < S) {
            const int p = parent_of(a, s);
            const int before = p < 0 ? 0 : length_of(a, p);
            more[r] = a.more[s];
            len[r] = (int)max((i64)before + min(more[r], 0), (i64)0);
            had = pages_of(a, before);
            has = pages_of(a, len[r]);
        }
        // A few pages a lane by itself, side by side; rows that give more a wave at a time.  (4000 sequences, all rows that way:
        // 41 us a call, so 33.)
        gave |= __any(had > has);
        constexpr int FEW = 4;
#pragma unroll
        for (int k = 0; k < FEW; ++k) {
            if (has + k >= had) break;
            int32_t *const at = a.t.d_page_table + (i64)s * W + has + k;
            const int page = *at;
            if (is_page(a, page)) atomicSub(&refs[page], 1);
            *at = -1;
        }
        has += FEW;
        unsigned long long rows = __ballot(had > has);
        while (rows) {
            const int l = __builtin_ctzll(rows);
            rows &= rows - 1;
            const int from = __builtin_amdgcn_readlane(has, l), to = __builtin_amdgcn_readlane(had, l);
            int32_t *const row = a.t.d_page_table + (i64)(r * kThreads + (tid & ~63) + l) * W;
            for (int c = from + lane; c < to; c += 64) {
                const int page = row[c];
                if (is_page(a, page)) atomicSub(&refs[page], 1);
                row[c] = -1;
            }
        }
    }
    if (__syncthreads_or(gave)) {
        __threadfence();
        __syncthreads();
        load_counts(0);
    }

    // who asks for what
    uint32_t tokens = 0, pages = 0;
    bool refused = false;                            // there are more tokens than the batch takes
    int start[ROWS] = {};
    for (int again = 0; again < 2; ++again) {
        tokens = pages = 0;
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const int s = r * kThreads + tid;
            if (r * kThreads >= S) break;
            bool wants = s < S && more[r] > 0 && (i64)len[r] + more[r] <= a.most;
            if (refused) wants = wants && plus(start[r], more[r]) <= (uint32_t)a.t.max_tokens;
            last[r] = -1;
            need[r] = 0;
            if (wants) {
                if (len[r] & (P - 1)) {
                    const int page = a.t.d_page_table[(i64)s * W + (len[r] >> a.page_shift)];
                    if (is_page(a, page) && __hip_atomic_load(&refs[page], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) > 1) last[r] = page;
                }
                need[r] = pages_of(a, len[r] + more[r]) - pages_of(a, len[r]) + (last[r] >= 0);
            }
            more[r] = wants ? more[r] : 0;
            const uint32_t v[2] = {(uint32_t)more[r], (uint32_t)need[r]};
            InFront f[2];
            in_front(v, waves, f);
            start[r] = (int)min(plus(tokens, f[0].before), (uint32_t)INT32_MAX);
            tokens = plus(tokens, f[0].all);
            if (s < S) {
                base[s] = (int)min(plus(pages, f[1].before), (uint32_t)INT32_MAX);
                const int c = pages_of(a, len[r]) - (last[r] >= 0);
                column[s] = last[r] >= 0 ? ~c : c;
            }
            pages = plus(pages, f[1].all);
        }
        if (refused || tokens <= (uint32_t)a.t.max_tokens) break;
        refused = true;      // once more: what those need that are turned away does not count
    }
    bool copies = false;
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
        if (r * kThreads < S) copies |= last[r] >= 0;
    copies = __syncthreads_or(copies);

    // free pages, in order, to who needs them
    uint32_t found = 0;
    for (i64 p0 = 0; p0 < a.t.num_pages && found < pages; p0 += kThreads * EACH) {
        if (p0) load_counts(p0);
        const i64 mine = p0 + tid * EACH;
        uint32_t free = 0;
#pragma unroll
        for (int q = 0; q < EACH / 4; ++q) {
            const int4 v = counts[q];
            free |= ((v.x == 0) | (v.y == 0) << 1 | (v.z == 0) << 2 | (v.w == 0) << 3) << 4 * q;
        }
        const uint32_t v[1] = {(uint32_t)__popc(free)};
        InFront f[1];
        in_front(v, waves, f);
        uint32_t rank = found + f[0].before;
        found += f[0].all;
        int s = free && rank < pages ? last_upto(base, S, (int)rank) : 0;
        for (; free && rank < pages; ++rank, free &= free - 1) {
            const int page = (int)mine + __builtin_ctz(free);
            while (s + 1 < S && base[s + 1] <= (int)rank) ++s;
            const int j = (int)rank - base[s], c = column[s];
            a.t.d_page_table[(i64)s * W + (c < 0 ? ~c : c) + j] = page;
            refs[page] = 1;
        }
    }
    // What was handed out is read again where pages ran out, or for a copy: only then it has to be in memory first.  (300 prompts, a
    // fence in any case: 13.4 us, so 10.4.)
    if (pages && (copies || found < pages)) __threadfence();
    __syncthreads();

    // who got it
    uint32_t total = 0;
    const bool all_served = !refused && found >= pages;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const int s = r * kThreads + tid;
        if (r * kThreads >= S) break;
        const bool served = s < S && more[r] > 0 && (need[r] == 0 || (i64)base[s] + need[r] <= (i64)found);
        if (s < S && need[r] > 0) {
            int32_t *const at = a.t.d_page_table + (i64)s * W + (column[s] < 0 ? ~column[s] : column[s]);
            if (served) {
                if (last[r] >= 0) {
                    a.t.d_copies[3 * s] = last[r];
                    a.t.d_copies[3 * s + 1] = at[0];
                    a.t.d_copies[3 * s + 2] = len[r] & (P - 1);
                    atomicSub(&refs[last[r]], 1);
                }
            } else {
                for (i64 j = 0; j < (i64)found - base[s]; ++j) {      // (one sequence at most: the pages ended within what it needs)
                    refs[at[j]] = 0;
                    at[j] = j == 0 && last[r] >= 0 ? last[r] : -1;
                }
            }
        }
        if (s < S && !(served && last[r] >= 0)) a.t.d_copies[3 * s] = a.t.d_copies[3 * s + 1] = a.t.d_copies[3 * s + 2] = -1;
        const int taken = served ? more[r] : 0;
        if (!all_served) {
            const uint32_t v[1] = {(uint32_t)taken};
            InFront f[1];
            in_front(v, waves, f);
            start[r] = (int)(total + f[0].before);
            total += f[0].all;
        }
        if (s < S) {
            a.t.d_seq_len[s] = len[r] + taken;
            a.t.d_taken[s] = taken;
            a.t.d_seq_start[s] = start[r];
            base[s] = start[r];      // (its own entries alone are looked at in this loop)
            column[s] = len[r] - start[r];
        }
    }
    if (all_served) total = tokens;
    if (tid == 0) a.t.d_seq_start[S] = (int)total;
    if (a.t.max_tokens > kFewTokens) return;
    __syncthreads();
    fill_tokens(a, base, column, (int)total, tid, kThreads);
}

__global__ __launch_bounds__(256) void k_tokens(AdvanceArgs a)
{
    __shared__ int start[kMostSeqs], shift[kMostSeqs];
    const int total = a.t.d_seq_start[a.t.num_seqs];
    for (int i = threadIdx.x; i < a.t.num_seqs; i += 256) {
        start[i] = a.t.d_seq_start[i];
        shift[i] = a.t.d_seq_len[i] - a.t.d_taken[i] - start[i];
    }
    __syncthreads();
    fill_tokens(a, start, shift, total, blockIdx.x * 256 + threadIdx.x, gridDim.x * 256);
}

// ---- copies of pages ----------------------------------------------------------------------------

// Workgroups (sequence, keys or values, part): a thread takes 16 bytes at a time.  (Bound by the launch: 192 pages of up to 16 keys
// of 4 heads of 128 in bf16 4.4 us.)
__global__ __launch_bounds__(256) void k_copy(CopyArgs a)
{
    const int s = blockIdx.x, parts = gridDim.z;
    const int64_t from = a.copies[3 * s], to = a.copies[3 * s + 1];
    const int slots = min(a.copies[3 * s + 2], 1 << a.cache.page_shift);
    if (from < 0 || from >= a.cache.num_pages || to < 0 || to >= a.cache.num_pages || slots <= 0) return;
    const int size = a.cache.k_scale ? 1 : 2, pieces = a.bytes / 16;
    uint8_t *const pool = (uint8_t *)(blockIdx.y ? a.cache.v : a.cache.k);
    const int64_t all = (int64_t)slots * a.kv_heads * pieces;
    for (int64_t i = blockIdx.z * 256 + threadIdx.x; i < all; i += parts * 256) {
        const int64_t at = i / pieces / a.kv_heads * a.cache.slot_stride + i / pieces % a.kv_heads * a.cache.head_stride;
        const int64_t byte = at * size + i % pieces * 16;
        *(uint4 *)(pool + to * a.cache.page_stride * size + byte) = *(const uint4 *)(pool + from * a.cache.page_stride * size + byte);
    }
    if (a.cache.k_scale) {
        uint8_t *const scale = blockIdx.y ? a.cache.v_scale : a.cache.k_scale;
        const int64_t blocks = (int64_t)(((slots - 1) >> a.cache.block_shift) + 1) * a.kv_heads;
        for (int64_t i = blockIdx.z * 256 + threadIdx.x; i < blocks; i += parts * 256) {
            const int64_t at = i / a.kv_heads * a.cache.scale_block_stride + i % a.kv_heads * a.cache.scale_head_stride;
            scale[to * a.cache.scale_page_stride + at] = scale[from * a.cache.scale_page_stride + at];
        }
    }
}

}  // namespace

hipError_t launch_advance(const AdvanceArgs &a, hipStream_t s)
{
    if (a.parent) {
        // (64 workgroups and more where the table is wide enough, of 16 columns at most)
        const int columns = std::max(1, std::min({16, kCells / a.t.num_seqs, a.t.table_width / 64}));
        k_reparent<<<std::min(4096, (a.t.table_width - 1) / columns + 1), kThreads, 0, s>>>(a, columns);
        if (hipError_t e = hipGetLastError()) return e;
    }
    if (a.t.num_seqs <= kThreads) k_advance<1><<<1, kThreads, 0, s>>>(a);
    else k_advance<kMostSeqs / kThreads><<<1, kThreads, 0, s>>>(a);
    if (hipError_t e = hipGetLastError()) return e;
    if (a.t.max_tokens > kFewTokens) {
        k_tokens<<<std::min(1024, (a.t.max_tokens - 1) / 256 + 1), 256, 0, s>>>(a);
        return hipGetLastError();
    }
    return hipSuccess;
}

hipError_t launch_copy(const CopyArgs &a, hipStream_t s)
{
    const int64_t most = ((int64_t)1 << a.cache.page_shift) * a.kv_heads * (a.bytes / 16);
    const dim3 grid((unsigned)a.num_seqs, 2, (unsigned)std::max<int64_t>(1, std::min<int64_t>(16, most / 2048)));
    k_copy<<<grid, 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace infaas
