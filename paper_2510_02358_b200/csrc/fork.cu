// dsp_cache_fork: new block tables from old ones, with shared blocks (rules: dsp.h).
//
// Who holds a block is found anew from the tables of the call, so nothing is kept between calls and dsp_cache_plan needs no counts:
//   0. every block that an input row holds is set to "nobody's";
//   1. every kept entry marks its block: -1 where the row keeps all of it, else the lowest row that keeps a part (a minimum, so the
//      order does not matter); every input entry marks the first place that names the block;
//   2. each output row sees whether its partly filled block is its own, each input row counts the blocks that nobody holds;
//   3. two prefix sums over the rows (formed by every CTA) give the places in the ring; tables and lists are written.
// A warp takes a row at a time.  Few table entries: one CTA runs the four parts with barriers between; many: four launches, each started
// early and waiting for the one before.
#include "dsp_common.cuh"

namespace dsp {
namespace {

constexpr int kNobody = 0x7FFFFFFF;
constexpr long long kOneCtaSteps = 32 * 16;      // rows times warp-wide table reads up to which one CTA is taken

struct ForkArgs {
    const int32_t *src, *keep;
    int Bo;
    const int32_t *seq_in, *count_in;
    const int64_t *pos_in;
    const int32_t *table_in;
    long long stride_in;
    int Bi, page, n_blocks, width;
    int32_t *ring, *table;
    long long stride;
    int32_t *count, *seq;
    int64_t *pos;
    int32_t *copy_src, *copy_dst, *copy_len;
    uint32_t *status;
    // workspace
    int32_t *holder, *first;         // [n_blocks]
    uint32_t *bad;                   // [Bo]
    int32_t *need, *back;            // [Bo], [Bi]
};

// The warps that work together, numbered through, and this one.
struct Crew {
    int warp, warps;
};

struct Row {
    int src, keep, n, full;          // blocks kept, of which full
    uint32_t status;
    __device__ __forceinline__ Row(const ForkArgs &a, int r) {
        src = a.src[r];
        keep = n = full = 0;
        status = 0u;
        if (src == -1) return;
        if (src < -1 || src >= a.Bi) { status = DSP_ROW_BAD_LENGTH; src = -1; return; }
        const int seq = a.seq_in[src];
        const int want = a.keep ? a.keep[r] : seq;
        const int have = min(max(a.count_in[src], 0), a.width);
        const int blocks = want > 0 ? (want - 1) / a.page + 1 : 0;
        if (seq < 0 || want < 0 || want > seq || blocks > have) { status = DSP_ROW_BAD_LENGTH; src = -1; return; }
        keep = want;
        n = blocks;
        full = want / a.page;
    }
};
__device__ __forceinline__ int held(const ForkArgs &a, int b) { return min(max(a.count_in[b], 0), a.width); }
__device__ __forceinline__ bool is_block(const ForkArgs &a, int p) { return p >= 0 && p < a.n_blocks; }
__device__ __forceinline__ void store_whole(int32_t *p) { asm volatile("st.relaxed.gpu.global.s32 [%0], %1;" ::"l"(p), "r"(-1) : "memory"); }

__device__ void part0(const ForkArgs &a, Crew c, int lane) {
    for (int b = c.warp; b < a.Bi; b += c.warps) {
        const int32_t *t = a.table_in + b * a.stride_in;
        for (int e = lane; e < held(a, b); e += 32)
            if (is_block(a, t[e])) {
                a.holder[t[e]] = kNobody;
                a.first[t[e]] = kNobody;
            }
    }
    for (int r = c.warp; r < a.Bo; r += c.warps) {
        const Row row(a, r);
        bool bad = false;
        for (int e = lane; e < row.n; e += 32) bad |= !is_block(a, a.table_in[row.src * a.stride_in + e]);
        if (__any_sync(0xFFFFFFFFu, bad) && lane == 0) a.bad[r] = DSP_ROW_BAD_BLOCK;
        else if (lane == 0) a.bad[r] = row.status;
    }
}

__device__ void part1(const ForkArgs &a, Crew c, int lane) {
    for (int r = c.warp; r < a.Bo; r += c.warps) {
        if (__ldcg(&a.bad[r])) continue;
        const Row row(a, r);
        const int32_t *t = a.table_in + row.src * a.stride_in;
        for (int e = lane; e < row.n; e += 32) {
            if (e < row.full) store_whole(&a.holder[t[e]]);
            else atomicMin(&a.holder[t[e]], r);
        }
    }
    for (int b = c.warp; b < a.Bi; b += c.warps) {
        const int32_t *t = a.table_in + b * a.stride_in;
        for (int e = lane; e < held(a, b); e += 32)
            if (is_block(a, t[e])) atomicMin(&a.first[t[e]], b * a.width + e);
    }
}

// Does entry e of input row b go back to the ring?
__device__ __forceinline__ bool goes_back(const ForkArgs &a, int b, int e, int p) {
    return is_block(a, p) && __ldcg(&a.holder[p]) == kNobody && __ldcg(&a.first[p]) == b * a.width + e;
}

__device__ void part2(const ForkArgs &a, Crew c, int lane) {
    for (int b = c.warp; b < a.Bi; b += c.warps) {
        const int32_t *t = a.table_in + b * a.stride_in;
        const int n = held(a, b);
        int back = 0;
        for (int e0 = 0; e0 < n; e0 += 32) {
            const int e = e0 + lane;
            back += __popc(__ballot_sync(0xFFFFFFFFu, e < n && goes_back(a, b, e, t[e])));
        }
        if (lane == 0) a.back[b] = back;
    }
    for (int r = c.warp * 32 + lane; r < a.Bo; r += c.warps * 32) {
        int need = 0;
        if (!__ldcg(&a.bad[r])) {
            const Row row(a, r);
            if (row.n > row.full) need = __ldcg(&a.holder[a.table_in[row.src * a.stride_in + row.full]]) != r;
        }
        a.need[r] = need;
    }
}

// Exclusive prefix sums of v[0 .. n) in shared memory, and the total at [n]; every thread of the CTA.
__device__ void prefix(const int32_t *v, int n, int32_t *out) {
    __shared__ int s_warp[32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
    const int per = (n + blockDim.x - 1) / blockDim.x;
    const int i0 = min(tid * per, n), i1 = min(i0 + per, n);
    int sum = 0;
    for (int i = i0; i < i1; ++i) sum += __ldcg(&v[i]);
    int incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(0xFFFFFFFFu, incl, o);
        if (lane >= o) incl += up;
    }
    __syncthreads();
    if (lane == 31) s_warp[warp] = incl;
    __syncthreads();
    int before = 0, all = 0;
    for (int i = 0; i < warps; ++i) {
        if (i < warp) before += s_warp[i];
        all += s_warp[i];
    }
    int at = before + incl - sum;
    for (int i = i0; i < i1; ++i) {
        out[i] = at;
        at += __ldcg(&v[i]);
    }
    if (tid == 0) out[n] = all;
    __syncthreads();
}

// shared: Bo + 1 + Bi + 1 words
__device__ void part3(const ForkArgs &a, Crew c, int lane, int32_t *shared, bool first_cta) {
    int32_t *s_need = shared, *s_back = shared + a.Bo + 1;
    prefix(a.need, a.Bo, s_need);
    prefix(a.back, a.Bi, s_back);
    const long long head = a.pos_in[0], tail = a.pos_in[1];
    const int free_blocks = (int)max(0LL, min(tail - head, (long long)a.n_blocks));
    const uint32_t nb = (uint32_t)a.n_blocks;
    const uint32_t head_at = (uint32_t)((head % a.n_blocks + a.n_blocks) % a.n_blocks);
    const uint32_t tail_at = (uint32_t)((tail % a.n_blocks + a.n_blocks) % a.n_blocks);
    if (first_cta && threadIdx.x == 0) {
        a.pos[0] = head + min(s_need[a.Bo], free_blocks);
        a.pos[1] = tail + s_back[a.Bi];
    }
    for (int r = c.warp; r < a.Bo; r += c.warps) {
        uint32_t status = __ldcg(&a.bad[r]);
        Row row(a, r);
        const bool need = s_need[r + 1] > s_need[r];
        if (need && s_need[r] >= free_blocks) status = DSP_ROW_NO_BLOCKS;
        if (status) row.n = row.keep = 0;
        const int fresh = need && !status ? a.ring[(head_at + (uint32_t)s_need[r]) % nb] : -1;
        const int32_t *t = a.table_in + row.src * a.stride_in;
        int32_t *out = a.table + r * a.stride;
        for (int e = lane; e < row.n; e += 32) out[e] = fresh >= 0 && e == row.full ? fresh : t[e];
        if (lane == 0) {
            a.count[r] = row.n;
            a.seq[r] = row.keep;
            a.status[r] = status;
            a.copy_src[r] = fresh >= 0 ? t[row.full] : -1;
            a.copy_dst[r] = fresh >= 0 ? fresh : -1;
            a.copy_len[r] = fresh >= 0 ? row.keep - row.full * a.page : 0;
        }
    }
    for (int b = c.warp; b < a.Bi; b += c.warps) {
        if (s_back[b + 1] == s_back[b]) continue;
        const int32_t *t = a.table_in + b * a.stride_in;
        const int n = held(a, b);
        uint32_t at = (uint32_t)s_back[b];
        for (int e0 = 0; e0 < n; e0 += 32) {
            const int e = e0 + lane;
            const bool back = e < n && goes_back(a, b, e, t[e]);
            const unsigned m = __ballot_sync(0xFFFFFFFFu, back);
            if (back) a.ring[(tail_at + at + (uint32_t)__popc(m & ((1u << lane) - 1u))) % nb] = t[e];
            at += (uint32_t)__popc(m);
        }
    }
}

template <int P>
__global__ void __launch_bounds__(1024) fork_part_kernel(const ForkArgs a) {
    extern __shared__ int32_t s_rows[];
    grid_launch_dependents();
    const int lane = threadIdx.x & 31;
    const Crew c = {(int)((blockIdx.x * blockDim.x + threadIdx.x) >> 5), (int)((gridDim.x * blockDim.x) >> 5)};
    if (P > 0) grid_dependency_wait();
    if (P == 0) part0(a, c, lane);
    if (P == 1) part1(a, c, lane);
    if (P == 2) part2(a, c, lane);
    if (P == 3) part3(a, c, lane, s_rows, blockIdx.x == 0);
}

__global__ void __launch_bounds__(1024) fork_kernel(const ForkArgs a) {
    extern __shared__ int32_t s_rows[];
    const int lane = threadIdx.x & 31;
    const Crew c = {(int)(threadIdx.x >> 5), (int)(blockDim.x >> 5)};
    part0(a, c, lane);
    __threadfence();
    __syncthreads();
    part1(a, c, lane);
    __threadfence();
    __syncthreads();
    part2(a, c, lane);
    __threadfence();
    __syncthreads();
    part3(a, c, lane, s_rows, true);
}

struct ForkWs {
    size_t off_holder, off_first, off_bad, off_need, off_back, total;
};
ForkWs fork_ws(int Bi, int Bo, int n_blocks) {
    ForkWs w;
    size_t o = 0;
    w.off_holder = o; o += align_up((size_t)n_blocks * 4, 256);
    w.off_first = o;  o += align_up((size_t)n_blocks * 4, 256);
    w.off_bad = o;    o += align_up((size_t)Bo * 4, 256);
    w.off_need = o;   o += align_up((size_t)Bo * 4, 256);
    w.off_back = o;   o += align_up((size_t)Bi * 4, 256);
    w.total = align_up(o + 1, 256);
    return w;
}

constexpr int kForkShared = (2 * DSP_MAX_PLAN_ROWS + 2) * (int)sizeof(int32_t);

int32_t launch_fork(const ForkArgs &a, cudaStream_t st) {
    const size_t smem = ((size_t)a.Bo + a.Bi + 2) * sizeof(int32_t);
    if (smem > 40 * 1024) {
        static std::atomic<unsigned long long> done_one{0}, done_part{0};
        DSP_CUDA_TRY(allow_shared(fork_kernel, kForkShared, done_one));
        DSP_CUDA_TRY(allow_shared(fork_part_kernel<3>, kForkShared, done_part));
    }
    const long long rows = (long long)a.Bi + a.Bo;
    if (rows * ((a.width + 31) / 32) <= kOneCtaSteps) {
        fork_kernel<<<1, 1024, smem, st>>>(a);
    } else {
        constexpr int kTh = 256;
        long long grid = (rows + kTh / 32 - 1) / (kTh / 32);
        if (grid > 2 * 148) grid = 2 * 148;
        fork_part_kernel<0><<<(unsigned)grid, kTh, 0, st>>>(a);
        DSP_CUDA_TRY(cudaGetLastError());
        DSP_CUDA_TRY(launch_dependent(fork_part_kernel<1>, (unsigned)grid, kTh, 0, st, a, true));
        DSP_CUDA_TRY(launch_dependent(fork_part_kernel<2>, (unsigned)grid, kTh, 0, st, a, true));
        DSP_CUDA_TRY(launch_dependent(fork_part_kernel<3>, (unsigned)grid, kTh, smem, st, a, true));
    }
    DSP_CUDA_TRY(cudaGetLastError());
    return DSP_OK;
}

// Do two tables [n, width] share memory?
bool overlap(const int32_t *a, long long sa, long long na, const int32_t *b, long long sb, long long nb, int width) {
    if (na < 1 || nb < 1) return false;
    return a < b + (nb - 1) * sb + width && b < a + (na - 1) * sa + width;
}

}  // namespace
}  // namespace dsp

extern "C" int32_t dsp_cache_fork_workspace_bytes(int32_t B_in, int32_t B_out, int32_t n_blocks, size_t *bytes) {
    using namespace dsp;
    if (!bytes || B_in < 0 || B_out < 0 || n_blocks < 1) return DSP_ERR_INVALID_ARG;
    if (B_in > DSP_MAX_PLAN_ROWS || B_out > DSP_MAX_PLAN_ROWS) return DSP_ERR_UNSUPPORTED;
    *bytes = fork_ws(B_in, B_out, n_blocks).total;
    return DSP_OK;
}

extern "C" int32_t dsp_cache_fork(const int32_t *src_row, const int32_t *keep_len, int32_t B_out,
                                  const int32_t *seq_len_in, const int32_t *block_count_in, const int64_t *ring_pos_in,
                                  const int32_t *block_table_in, int64_t table_in_stride, int32_t B_in,
                                  int32_t page_size, int32_t n_blocks, int32_t max_blocks, int32_t *free_ring,
                                  int32_t *block_table, int64_t table_stride, int32_t *block_count, int32_t *seq_len,
                                  int64_t *ring_pos, int32_t *copy_src, int32_t *copy_dst, int32_t *copy_len,
                                  uint32_t *row_status, void *workspace, size_t workspace_bytes, dsp_stream_t stream) {
    using namespace dsp;
    if (B_in < 0 || B_out < 0 || page_size < 1 || n_blocks < 1 || max_blocks < 1) return DSP_ERR_INVALID_ARG;
    if (table_in_stride < max_blocks || table_stride < max_blocks) return DSP_ERR_INVALID_ARG;
    if (B_in > DSP_MAX_PLAN_ROWS || B_out > DSP_MAX_PLAN_ROWS) return DSP_ERR_UNSUPPORTED;
    if ((long long)(B_in > B_out ? B_in : B_out) * max_blocks > (1 << 30)) return DSP_ERR_UNSUPPORTED;
    if (!ring_pos_in || !ring_pos || !free_ring || !workspace) return DSP_ERR_INVALID_ARG;
    if (B_in > 0 && (!seq_len_in || !block_count_in || !block_table_in)) return DSP_ERR_INVALID_ARG;
    if (B_out > 0 && (!src_row || !block_table || !block_count || !seq_len || !copy_src || !copy_dst || !copy_len || !row_status))
        return DSP_ERR_INVALID_ARG;
    if (ring_pos == ring_pos_in || (B_out > 0 && (block_count == block_count_in || seq_len == seq_len_in))) return DSP_ERR_INVALID_ARG;
    if (overlap(block_table_in, table_in_stride, B_in, block_table, table_stride, B_out, max_blocks)) return DSP_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(workspace) & 255) != 0) return DSP_ERR_INVALID_ARG;
    const ForkWs w = fork_ws(B_in, B_out, n_blocks);
    if (workspace_bytes < w.total) return DSP_ERR_WORKSPACE;
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    ForkArgs a = {};
    a.src = src_row; a.keep = keep_len; a.Bo = B_out;
    a.seq_in = seq_len_in; a.count_in = block_count_in; a.pos_in = ring_pos_in;
    a.table_in = block_table_in; a.stride_in = table_in_stride; a.Bi = B_in;
    a.page = page_size; a.n_blocks = n_blocks; a.width = max_blocks;
    a.ring = free_ring; a.table = block_table; a.stride = table_stride;
    a.count = block_count; a.seq = seq_len; a.pos = ring_pos;
    a.copy_src = copy_src; a.copy_dst = copy_dst; a.copy_len = copy_len; a.status = row_status;
    a.holder = reinterpret_cast<int32_t *>(ws + w.off_holder);
    a.first = reinterpret_cast<int32_t *>(ws + w.off_first);
    a.bad = reinterpret_cast<uint32_t *>(ws + w.off_bad);
    a.need = reinterpret_cast<int32_t *>(ws + w.off_need);
    a.back = reinterpret_cast<int32_t *>(ws + w.off_back);
    return launch_fork(a, reinterpret_cast<cudaStream_t>(stream));
}
