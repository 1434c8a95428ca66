// dsp_cache_fork: new block tables from old ones, with shared blocks (rules: dsp.h).
//
// Who holds a block is found anew from the tables of the call, so nothing is kept between calls and dsp_cache_plan needs no counts:
//   0. every block is set to "nobody's";
//   1. every kept entry marks its block: -1 where the row keeps all of it, else the lowest row that keeps a part (a minimum, so the
//      order does not matter); every input entry marks the first place that names the block;
//   2. each output row sees whether its partly filled block is its own, each input row counts the blocks that nobody holds;
//   3. a prefix sum over the rows (formed by every CTA) gives the places in the ring; tables and lists are written.
// A warp takes a row at a time, with four table entries a lane under way.  Few rows and blocks: one CTA runs all parts, with the marks in
// shared memory and barriers between; many: a fill and three launches, each started early and waiting for the one before.
//
// The bytes are nothing (512 requests of 8192 tokens: 0.6 MB); what bounds the call is the chain of dependent reads (row, table, mark) in each
// part and the launches.  Measured: 4 requests 5.0 us, 16 7.6, 64 9.3, 500 10.6.
// A cluster of 16 CTAs instead of the fill and the launches: 512 requests of 8192 tokens 21 us instead of 15.
#include "dsp_common.cuh"

namespace dsp {
namespace {

constexpr int kNobody = 0x7F7F7F7F;              // what a fill with bytes leaves
// Rows (old and new ones) up to which one CTA is taken: two rounds of its 32 warps.  Measured (us, one CTA / launches): 4 + 4 rows of 500 tokens
// 5.0 / 10.3, 16 + 16 of 8000 12.8 / 27.8, 32 + 32 of 500 9.5 / 9.3, of 2000 10.3 / 12.2, 40 + 40 of 500 11.2 / 9.3, 64 + 64 13.2 / 9.5, 500 + 500 67 / 10.6.
constexpr long long kOneCtaRows = 64;
constexpr int kOneCtaShared = 200 * 1024;
constexpr int kPrefixWarps = 32;                 // of a CTA, at most: their sums lie in static shared memory
// Dynamic shared memory of a launch that has not asked for more: 48 KB with the kernel's static share in them.
constexpr int kSharedByDefault = 48 * 1024 - kPrefixWarps * 8;
constexpr int kU = 4;                            // entries a lane has under way

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
    // workspace (or shared memory)
    int32_t *holder, *first;         // [n_blocks]
    int4 *rows;                      // [Bo] input row, tokens kept, blocks kept, status
    int32_t *need, *back;            // [Bo], [Bi]
};

// The warps that work together, numbered through, and this one.
struct Crew {
    int warp, warps;
};

__device__ __forceinline__ int held(const ForkArgs &a, int b) { return min(max(a.count_in[b], 0), a.width); }
__device__ __forceinline__ bool is_block(const ForkArgs &a, int p) { return p >= 0 && p < a.n_blocks; }
__device__ __forceinline__ void store_whole(int32_t *p) { asm volatile("st.relaxed.gpu.s32 [%0], %1;" ::"l"(p), "r"(-1) : "memory"); }

// What row r asks for, its blocks not yet looked at.
__device__ __forceinline__ int4 asked(const ForkArgs &a, int r) {
    const int src = a.src[r];
    if (src == -1) return make_int4(-1, 0, 0, 0);
    const int4 bad = make_int4(-1, 0, 0, DSP_ROW_BAD_LENGTH);
    if (src < -1 || src >= a.Bi) return bad;
    const int seq = a.seq_in[src], have = held(a, src), want = a.keep ? a.keep[r] : seq;
    const int blocks = want > 0 ? (want - 1) / a.page + 1 : 0;
    if (seq < 0 || want < 0 || want > seq || blocks > have) return bad;
    return make_int4(src, want, blocks, 0);
}
__device__ __forceinline__ bool partly(const ForkArgs &a, const int4 &row) { return row.z > 0 && row.y % a.page != 0; }

// Calls see(e, block) for the first n entries of a table's row, a warp's lanes side by side (beyond n: block -1, e >= n).
template <typename See>
__device__ __forceinline__ void entries(const int32_t *t, int n, int lane, See see) {
    for (int e0 = lane; e0 - lane < n; e0 += 32 * kU) {
        int p[kU];
#pragma unroll
        for (int j = 0; j < kU; ++j) p[j] = e0 + 32 * j < n ? t[e0 + 32 * j] : -1;
#pragma unroll
        for (int j = 0; j < kU; ++j)
            if (e0 - lane + 32 * j < n) see(e0 + 32 * j, p[j]);
    }
}

__device__ void part1(const ForkArgs &a, Crew c, int lane) {
    for (int r = c.warp; r < a.Bo + a.Bi; r += c.warps) {
        if (r < a.Bo) {
            int4 row = asked(a, r);
            const int32_t *t = a.table_in + max(row.x, 0) * a.stride_in;
            bool bad = false;
            entries(t, row.z, lane, [&](int e, int p) { bad |= e < row.z && !is_block(a, p); });
            if (__any_sync(0xFFFFFFFFu, bad)) row = make_int4(-1, 0, 0, DSP_ROW_BAD_BLOCK);
            const int full = row.z - (partly(a, row) ? 1 : 0);
            entries(t, row.z, lane, [&](int e, int p) {
                if (e < full) store_whole(&a.holder[p]);
                else if (e < row.z) atomicMin(&a.holder[p], r);
            });
            if (lane == 0) a.rows[r] = row;
        } else {
            const int b = r - a.Bo;
            entries(a.table_in + b * a.stride_in, held(a, b), lane, [&](int e, int p) {
                if (is_block(a, p)) atomicMin(&a.first[p], b * a.width + e);
            });
        }
    }
}

template <typename T> __device__ __forceinline__ T fresh_load(const T *p) { return *const_cast<const volatile T *>(p); }
__device__ __forceinline__ int4 fresh_load(const int4 *p) {
    const volatile int *q = reinterpret_cast<const volatile int *>(p);
    return make_int4(q[0], q[1], q[2], q[3]);
}

__device__ __forceinline__ bool goes_back(const ForkArgs &a, int b, int e, int p) {
    return is_block(a, p) && fresh_load(&a.holder[p]) == kNobody && fresh_load(&a.first[p]) == b * a.width + e;
}

__device__ void part2(const ForkArgs &a, Crew c, int lane) {
    for (int b = c.warp; b < a.Bi; b += c.warps) {
        int back = 0;
        entries(a.table_in + b * a.stride_in, held(a, b), lane, [&](int e, int p) {
            back += __popc(__ballot_sync(0xFFFFFFFFu, goes_back(a, b, e, p)));
        });
        if (lane == 0) a.back[b] = back;
    }
    for (int r = c.warp * 32 + lane; r < a.Bo; r += c.warps * 32) {
        const int4 row = fresh_load(&a.rows[r]);
        a.need[r] = partly(a, row) && fresh_load(&a.holder[a.table_in[row.x * a.stride_in + row.z - 1]]) != r;
    }
}

// Exclusive prefix sums over the rows of the blocks needed (low half) and given back (high half): [n] holds the totals.  Every thread of the CTA.
__device__ void prefix(const ForkArgs &a, int n, unsigned long long *out) {
    __shared__ unsigned long long s_warp[kPrefixWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
    const int per = (n + blockDim.x - 1) / blockDim.x;
    const int i0 = min(tid * per, n), i1 = min(i0 + per, n);
    auto at_row = [&](int i) {
        const unsigned need = i < a.Bo ? (unsigned)fresh_load(&a.need[i]) : 0u, back = i < a.Bi ? (unsigned)fresh_load(&a.back[i]) : 0u;
        return (unsigned long long)back << 32 | need;
    };
    unsigned long long sum = 0, incl;
    for (int i = i0; i < i1; ++i) {
        const unsigned long long v = at_row(i);
        out[i] = sum;                            // within the thread's share at first
        sum += v;
    }
    incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned long long up = __shfl_up_sync(0xFFFFFFFFu, incl, o);
        if (lane >= o) incl += up;
    }
    if (lane == 31) s_warp[warp] = incl;
    __syncthreads();
    unsigned long long before = 0, all = 0;
    for (int i = 0; i < warps; ++i) {
        if (i < warp) before += s_warp[i];
        all += s_warp[i];
    }
    before += incl - sum;
    for (int i = i0; i < i1; ++i) out[i] += before;
    if (tid == 0) out[n] = all;
    __syncthreads();
}

// shared: max(Bo, Bi) + 1 numbers of 64 bits
__device__ void part3(const ForkArgs &a, Crew c, int lane, unsigned long long *sums, bool first_cta) {
    const int n = max(a.Bo, a.Bi);
    const long long head = a.pos_in[0], tail = a.pos_in[1];
    prefix(a, n, sums);
    const int free_blocks = (int)max(0LL, min(tail - head, (long long)a.n_blocks));
    const uint32_t nb = (uint32_t)a.n_blocks;
    const uint32_t head_at = (uint32_t)((head % a.n_blocks + a.n_blocks) % a.n_blocks);
    const uint32_t tail_at = (uint32_t)((tail % a.n_blocks + a.n_blocks) % a.n_blocks);
    if (first_cta && threadIdx.x == 0) {
        a.pos[0] = head + min((int)(uint32_t)sums[n], free_blocks);
        a.pos[1] = tail + (long long)(sums[n] >> 32);
    }
    for (int r = c.warp; r < a.Bo + a.Bi; r += c.warps) {
        if (r < a.Bo) {
            int4 row = fresh_load(&a.rows[r]);
            const int rank = (int)(uint32_t)sums[r];
            const bool need = (uint32_t)sums[r + 1] != (uint32_t)sums[r];
            if (need && rank >= free_blocks) row = make_int4(-1, 0, 0, DSP_ROW_NO_BLOCKS);
            const bool copies = need && row.w == 0;
            const int fresh = copies ? a.ring[(head_at + (uint32_t)rank) % nb] : -1, last = row.z - 1;
            int32_t *out = a.table + r * a.stride;
            entries(a.table_in + max(row.x, 0) * a.stride_in, row.z, lane, [&](int e, int p) {
                if (e >= row.z) return;
                out[e] = copies && e == last ? fresh : p;
                if (e == last) a.copy_src[r] = copies ? p : -1;
            });
            if (lane == 0) {
                a.count[r] = row.z;
                a.seq[r] = row.y;
                a.status[r] = (uint32_t)row.w;
                if (row.z == 0) a.copy_src[r] = -1;
                a.copy_dst[r] = fresh;
                a.copy_len[r] = copies ? row.y - last * a.page : 0;
            }
        } else {
            const int b = r - a.Bo;
            uint32_t at = (uint32_t)(sums[b] >> 32);
            if ((uint32_t)(sums[b + 1] >> 32) == at) continue;
            entries(a.table_in + b * a.stride_in, held(a, b), lane, [&](int e, int p) {
                const bool back = goes_back(a, b, e, p);
                const unsigned m = __ballot_sync(0xFFFFFFFFu, back);
                if (back) a.ring[(tail_at + at + (uint32_t)__popc(m & ((1u << lane) - 1u))) % nb] = p;
                at += (uint32_t)__popc(m);
            });
        }
    }
}

template <int P>
__global__ void __launch_bounds__(256) fork_part_kernel(const ForkArgs a) {
    extern __shared__ __align__(16) unsigned long long s_sums[];
    grid_launch_dependents();
    const int lane = threadIdx.x & 31;
    const Crew c = {(int)((blockIdx.x * blockDim.x + threadIdx.x) >> 5), (int)((gridDim.x * blockDim.x) >> 5)};
    grid_dependency_wait();
    if (P == 1) part1(a, c, lane);
    if (P == 2) part2(a, c, lane);
    if (P == 3) part3(a, c, lane, s_sums, blockIdx.x == 0);
}

// Shared memory of the one CTA: the sums, the rows, the numbers of a row, the marks.
__host__ __device__ inline long long one_cta_bytes(int Bi, int Bo, int n_blocks) {
    const long long n = Bi > Bo ? Bi : Bo;
    return 16 * Bo + 8 * ((n + 2) & ~1ll) + 4ll * (Bo + Bi) + 8ll * n_blocks;
}
__global__ void __launch_bounds__(1024) fork_kernel(const ForkArgs in) {
    extern __shared__ __align__(16) unsigned char s_all[];
    const int lane = threadIdx.x & 31, n = max(in.Bi, in.Bo);
    const Crew c = {(int)(threadIdx.x >> 5), (int)(blockDim.x >> 5)};
    ForkArgs a = in;
    a.rows = reinterpret_cast<int4 *>(s_all);
    unsigned long long *sums = reinterpret_cast<unsigned long long *>(a.rows + a.Bo);
    a.need = reinterpret_cast<int32_t *>(sums + ((n + 2) & ~1));
    a.back = a.need + a.Bo;
    a.holder = a.back + a.Bi;
    a.first = a.holder + a.n_blocks;
    for (int i = threadIdx.x; i < 2 * a.n_blocks; i += blockDim.x) a.holder[i] = kNobody;
    __syncthreads();
    part1(a, c, lane);
    __syncthreads();
    part2(a, c, lane);
    __syncthreads();
    part3(a, c, lane, sums, true);
}

struct ForkWs {
    size_t off_marks, mark_bytes, off_first, off_rows, off_need, off_back, total;
};
ForkWs fork_ws(int Bi, int Bo, int n_blocks) {
    ForkWs w;
    size_t o = 0;
    w.off_marks = o;  o += align_up((size_t)n_blocks * 4, 256);
    w.off_first = o;  o += align_up((size_t)n_blocks * 4, 256);
    w.mark_bytes = o;
    w.off_rows = o;   o += align_up((size_t)Bo * 16, 256);
    w.off_need = o;   o += align_up((size_t)Bo * 4, 256);
    w.off_back = o;   o += align_up((size_t)Bi * 4, 256);
    w.total = o;
    return w;
}

int32_t launch_fork(const ForkArgs &a, size_t mark_bytes, cudaStream_t st) {
    const long long rows = (long long)a.Bi + a.Bo;
    const long long one = one_cta_bytes(a.Bi, a.Bo, a.n_blocks);
    if (rows <= kOneCtaRows && one <= kOneCtaShared) {
        static std::atomic<unsigned long long> done{0};
        if (one > kSharedByDefault) DSP_CUDA_TRY(allow_shared(fork_kernel, kOneCtaShared, done));
        const unsigned threads = rows <= 8 ? 256u : 1024u;       // a warp for each row
        fork_kernel<<<1, threads, (size_t)one, st>>>(a);
    } else {
        static std::atomic<unsigned long long> done{0};
        const size_t smem = ((size_t)(a.Bi > a.Bo ? a.Bi : a.Bo) + 1) * 8;
        if (smem > kSharedByDefault) DSP_CUDA_TRY(allow_shared(fork_part_kernel<3>, (DSP_MAX_PLAN_ROWS + 1) * 8, done));
        constexpr int kTh = 256;
        long long grid = (rows + kTh / 32 - 1) / (kTh / 32);
        grid = grid < 1 ? 1 : grid > 4 * 148 ? 4 * 148 : grid;   // without rows the ring's ends are handed on
        DSP_CUDA_TRY(cudaMemsetAsync(a.holder, kNobody & 0xFF, mark_bytes, st));
        fork_part_kernel<1><<<(unsigned)grid, kTh, 0, st>>>(a);
        DSP_CUDA_TRY(cudaGetLastError());
        DSP_CUDA_TRY(launch_dependent(fork_part_kernel<2>, (unsigned)grid, kTh, 0, st, a, true));
        DSP_CUDA_TRY(launch_dependent(fork_part_kernel<3>, (unsigned)grid, kTh, smem, st, a, true));
    }
    DSP_CUDA_TRY(cudaGetLastError());
    return DSP_OK;
}

// Do two tables [n, width] share memory?  The rows of one may lie in the gaps of the other (two halves of a wider tensor).
bool overlap(const int32_t *a, long long sa, long long na, const int32_t *b, long long sb, long long nb, int width) {
    if (na < 1 || nb < 1) return false;
    // entries from the start of b to that of a's row i; rows of b begin every sb
    const long long between = (long long)(reinterpret_cast<intptr_t>(a) - reinterpret_cast<intptr_t>(b)) / (long long)sizeof(int32_t);
    const long long end = (nb - 1) * sb + width;
    if (between >= end || between + (na - 1) * sa + width <= 0) return false;
    for (long long i = 0; i < na; ++i) {
        const long long at = between + i * sa;
        if (at + width <= 0 || at >= end) continue;
        const long long row = at < 0 ? 0 : at / sb, past = at - row * sb;    // the last row of b that begins at or before `at`, or the first
        if (past < width) return true;
        if (row + 1 < nb && sb - past < width) return true;
    }
    return false;
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
    a.holder = reinterpret_cast<int32_t *>(ws + w.off_marks);
    a.first = reinterpret_cast<int32_t *>(ws + w.off_first);
    a.rows = reinterpret_cast<int4 *>(ws + w.off_rows);
    a.need = reinterpret_cast<int32_t *>(ws + w.off_need);
    a.back = reinterpret_cast<int32_t *>(ws + w.off_back);
    return launch_fork(a, w.mark_bytes, reinterpret_cast<cudaStream_t>(stream));
}
