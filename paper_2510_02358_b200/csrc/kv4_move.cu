// dsp_kv4_copy, dsp_kv4_compact: bytes of the 4-bit cache move, for all layers of a model in one launch.
//
// A copy of a block is one piece of memory a head (the runs up to the copied tokens); a warp moves a run, 16 bytes a lane.  A token is no
// such piece: its codes are cut into the places of a matrix instruction's fragments (kv4.cuh), D / 4 words of 4 bytes and its scales and
// offsets.  The same lane always takes the same word of a token, so the moves of a request need no barrier: a lane's reads and writes of
// one address come in its own order, and since the accepted nodes grow along the path no target lies behind a later source.
//
// Both are bound by latency, not by their bytes: 96 forks of 8704-byte heads in 4 layers 9.5 us with the launch, 64 trees of up to 16 accepted nodes in 16
// layers of 8 heads 9.4 us (7 MB, 1.1 us at a copy's rate), one tree 4.6 us.  A warp a head for a tree: 8192 warps, each with a chain of table, node
// and word reads; a warp a block and head instead of a run and head for the copies: 11.5 us.
#include "kv4.cuh"

namespace dsp {
namespace {

constexpr int kMoveThreads = 256;

struct CopyArgs {
    uint8_t *cache;
    long long layer_stride, head_bytes;      // bytes from layer to layer; of one head of one block
    int layers, n_blocks, page, Hkv, runs;   // runs of a block
    const int32_t *src, *dst, *len;
    int N;
};

// A unit is a run of 16 tokens of an entry, layer and head.  A warp looks at 32 units at a time, which lie a grid apart, and copies those
// that count, each with all of its reads under way at once.
template <int D>
__global__ void __launch_bounds__(kMoveThreads) kv4_copy_kernel(const CopyArgs a) {
    constexpr int kVecs = Kv4<D>::kRunBytes / 16, kU = (kVecs + 31) / 32;
    const int lane = threadIdx.x & 31;
    const long long warp = ((long long)blockIdx.x * kMoveThreads + threadIdx.x) >> 5, warps = ((long long)gridDim.x * kMoveThreads) >> 5;
    const long long per = (long long)a.layers * a.Hkv * a.runs, units = a.N * per;
    for (long long u0 = warp; u0 < units; u0 += warps * 32) {
        const long long u = u0 + warps * lane;
        const uint8_t *from = nullptr;
        uint8_t *to = nullptr;
        if (u < units) {
            const int i = (int)(u / per);
            const unsigned rest = (unsigned)(u - i * per), unit = rest / (unsigned)a.runs;
            const int run = (int)(rest - unit * (unsigned)a.runs), layer = (int)(unit / (unsigned)a.Hkv), h = (int)unit - layer * a.Hkv;
            const int s = a.src[i], d = a.dst[i], n = a.len ? a.len[i] : a.page;
            if (s >= 0 && s < a.n_blocks && d >= 0 && d < a.n_blocks && run * 16 < n) {
                uint8_t *base = a.cache + layer * a.layer_stride + (long long)run * Kv4<D>::kRunBytes;
                from = base + ((long long)s * a.Hkv + h) * a.head_bytes;
                to = base + ((long long)d * a.Hkv + h) * a.head_bytes;
            }
        }
        unsigned some = __ballot_sync(0xFFFFFFFFu, from != nullptr);
        while (some) {
            const int k = __ffs(some) - 1;
            some &= some - 1;
            const uint4 *p = reinterpret_cast<const uint4 *>(__shfl_sync(0xFFFFFFFFu, reinterpret_cast<unsigned long long>(from), k)) + lane;
            uint4 *q = reinterpret_cast<uint4 *>(__shfl_sync(0xFFFFFFFFu, reinterpret_cast<unsigned long long>(to), k)) + lane;
            uint4 r[kU];
#pragma unroll
            for (int j = 0; j < kU; ++j)
                if (lane + 32 * j < kVecs) r[j] = p[32 * j];
#pragma unroll
            for (int j = 0; j < kU; ++j)
                if (lane + 32 * j < kVecs) q[32 * j] = r[j];
        }
    }
}

struct CompactArgs {
    uint8_t *cache;
    long long layer_stride;
    int layers, n_blocks, page, Hkv;
    const int32_t *table;
    long long table_stride;
    int width;
    const int32_t *seq, *node, *len;
    int B, L;
};

// A warp for a head of a layer of a request.
template <int D>
__global__ void __launch_bounds__(kMoveThreads) kv4_compact_kernel(const CompactArgs a) {
    using F = Kv4<D>;
    constexpr int kWords = D / 8;                        // of a key, and of a value
    const int lane = threadIdx.x & 31;
    const long long unit = ((long long)blockIdx.x * kMoveThreads + threadIdx.x) >> 5;
    const int per = a.layers * a.Hkv;
    const int b = (int)(unit / per);
    if (b >= a.B) return;
    const int rest = (int)(unit - (long long)b * per), layer = rest / a.Hkv, h = rest - layer * a.Hkv;
    const int n = min(max(a.len[b], 0), a.L);
    const long long start = (long long)a.seq[b] + 1;
    uint8_t *cache = a.cache + layer * a.layer_stride;
    const int runs = a.page / 16;
    // byte of the run that holds a position of the request, in this head (-1: nowhere), and the token's place in it
    auto run_of = [&](long long at) -> long long {
        const long long e = at / a.page;
        if (at < 0 || e >= a.width) return -1;
        const int block = a.table[b * a.table_stride + e];
        if (block < 0 || block >= a.n_blocks) return -1;
        return (((long long)block * a.Hkv + h) * runs + (at - e * a.page) / 16) * F::kRunBytes;
    };
    const bool key = lane < kWords, value = lane >= kWords && lane < 2 * kWords;
    auto word_of = [&](int t) { return key ? F::key_word(t, lane) : F::kValueOff + F::value_word(t, lane - kWords); };
    for (int i0 = 0; i0 < n; i0 += 32) {
        const int i = i0 + lane;
        const int node = i < n ? a.node[(long long)b * a.L + i] : -1;
        long long from = -1, to = -1;
        int places = 0;
        if (node >= 0 && node != i) {
            from = run_of(start + node);
            to = run_of(start + i);
            places = (int)((start + node) % a.page % 16) | (int)((start + i) % a.page % 16) << 8;
        }
        unsigned some = __ballot_sync(0xFFFFFFFFu, from >= 0 && to >= 0);
        while (some) {
            constexpr int kU = 4;                        // tokens under way together: read before any of them is written
            uint32_t w[kU], par[kU];
            uint8_t *q[kU];
            int t[kU];
#pragma unroll
            for (int j = 0; j < kU; ++j) {
                q[j] = nullptr;
                if (!some) continue;                     // the warp alike
                const int k = __ffs(some) - 1;
                some &= some - 1;
                const uint8_t *p = cache + __shfl_sync(0xFFFFFFFFu, from, k);
                q[j] = cache + __shfl_sync(0xFFFFFFFFu, to, k);
                const int pl = __shfl_sync(0xFFFFFFFFu, places, k);
                t[j] = pl >> 8;
                if (key || value) w[j] = *reinterpret_cast<const uint32_t *>(p + word_of(pl & 15));
                if (lane < 2) par[j] = *reinterpret_cast<const uint32_t *>(p + F::kParamOff + (pl & 15) * 8 + lane * 4);
            }
#pragma unroll
            for (int j = 0; j < kU; ++j) {
                if (!q[j]) continue;
                if (key || value) *reinterpret_cast<uint32_t *>(q[j] + word_of(t[j])) = w[j];
                if (lane < 2) *reinterpret_cast<uint32_t *>(q[j] + F::kParamOff + t[j] * 8 + lane * 4) = par[j];
            }
        }
    }
}

int32_t check_layers(const void *cache, int32_t layers, int64_t layer_stride, int32_t n_blocks, int32_t page_size, int32_t Hkv, int32_t D) {
    if (layers < 1 || n_blocks < 1 || Hkv < 1 || page_size < 16 || page_size % 16 != 0) return DSP_ERR_INVALID_ARG;
    if ((D != 64 && D != 128) || layers > 65535 || Hkv > 4096) return DSP_ERR_UNSUPPORTED;
    if (!cache || (reinterpret_cast<uintptr_t>(cache) & 15) != 0) return DSP_ERR_INVALID_ARG;
    if (layers > 1 && (layer_stride % 16 != 0 || layer_stride / page_size / (D + 8) / Hkv < n_blocks)) return DSP_ERR_INVALID_ARG;
    return DSP_OK;
}

}  // namespace
}  // namespace dsp

extern "C" int32_t dsp_kv4_copy(void *cache, int32_t layers, int64_t layer_stride, int32_t n_blocks, int32_t page_size,
                                int32_t Hkv, int32_t D, const int32_t *copy_src, const int32_t *copy_dst,
                                const int32_t *copy_len, int32_t N, dsp_stream_t stream) {
    using namespace dsp;
    if (N < 0) return DSP_ERR_INVALID_ARG;
    const int32_t rc = check_layers(cache, layers, layer_stride, n_blocks, page_size, Hkv, D);
    if (rc != DSP_OK) return rc;
    if (N > (1 << 24)) return DSP_ERR_UNSUPPORTED;
    if (N == 0) return DSP_OK;
    if (!copy_src || !copy_dst) return DSP_ERR_INVALID_ARG;
    CopyArgs a = {};
    a.cache = static_cast<uint8_t *>(cache);
    a.layer_stride = layers > 1 ? layer_stride : 0;
    a.head_bytes = (long long)page_size * (D + 8);
    a.layers = layers; a.n_blocks = n_blocks; a.page = page_size; a.Hkv = Hkv; a.runs = page_size / 16;
    a.src = copy_src; a.dst = copy_dst; a.len = copy_len; a.N = N;
    if ((long long)layers * Hkv * a.runs > 0x7FFFFFFFLL) return DSP_ERR_UNSUPPORTED;
    const long long warps = (long long)N * layers * Hkv * a.runs;
    long long grid = (warps + kMoveThreads / 32 - 1) / (kMoveThreads / 32);
    if (grid > 148 * 4) grid = 148 * 4;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (D == 64) kv4_copy_kernel<64><<<(unsigned)grid, kMoveThreads, 0, st>>>(a);
    else kv4_copy_kernel<128><<<(unsigned)grid, kMoveThreads, 0, st>>>(a);
    DSP_CUDA_TRY(cudaGetLastError());
    return DSP_OK;
}

extern "C" int32_t dsp_kv4_compact(void *cache, int32_t layers, int64_t layer_stride, int32_t n_blocks, int32_t page_size,
                                   int32_t Hkv, int32_t D, const int32_t *block_table, int64_t table_stride, int32_t max_blocks,
                                   const int32_t *seq_len, const int32_t *accepted_node, const int32_t *accepted_len,
                                   int32_t B, int32_t L, dsp_stream_t stream) {
    using namespace dsp;
    if (B < 0 || L < 0 || max_blocks < 1 || table_stride < max_blocks) return DSP_ERR_INVALID_ARG;
    const int32_t rc = check_layers(cache, layers, layer_stride, n_blocks, page_size, Hkv, D);
    if (rc != DSP_OK) return rc;
    if (B > (1 << 24)) return DSP_ERR_UNSUPPORTED;
    if (B == 0 || L == 0) return DSP_OK;
    if (!block_table || !seq_len || !accepted_node || !accepted_len) return DSP_ERR_INVALID_ARG;
    CompactArgs a = {};
    a.cache = static_cast<uint8_t *>(cache);
    a.layer_stride = layers > 1 ? layer_stride : 0;
    a.layers = layers; a.n_blocks = n_blocks; a.page = page_size; a.Hkv = Hkv;
    a.table = block_table; a.table_stride = table_stride; a.width = max_blocks;
    a.seq = seq_len; a.node = accepted_node; a.len = accepted_len;
    a.B = B; a.L = L;
    const long long grid = ((long long)B * layers * Hkv + kMoveThreads / 32 - 1) / (kMoveThreads / 32);
    if (grid > 0x7FFFFFFFLL) return DSP_ERR_UNSUPPORTED;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (D == 64) kv4_compact_kernel<64><<<(unsigned)grid, kMoveThreads, 0, st>>>(a);
    else kv4_compact_kernel<128><<<(unsigned)grid, kMoveThreads, 0, st>>>(a);
    DSP_CUDA_TRY(cudaGetLastError());
    return DSP_OK;
}
