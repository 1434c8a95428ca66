// dsp_attn_kv4: attention of a step's tokens over the paged 4-bit cache.
#include <math.h>

#include "kv4.cuh"

namespace dsp {
namespace {

struct AttnArgs {
    const __nv_bfloat16 *q;
    long long q_t, q_h;
    int B, T, Hq, Hkv;
    const uint8_t *cache;
    int n_blocks, page;
    const int32_t *table;
    long long table_stride;
    int max_blocks;
    const int32_t *kv_len, *cu;
    int max_new;
    float scale;
    int mask_kind;
    const uint32_t *bits;
    int words;
    __nv_bfloat16 *out;
};

// One warp per token and query head, one cached token after the other.
template <int D>
__global__ void __launch_bounds__(128) attn_simple_kernel(const AttnArgs a) {
    constexpr int kCh = D / 32;                                   // channels of a lane
    const int lane = threadIdx.x & 31;
    const long long unit = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    const int t = (int)(unit / a.Hq), h = (int)(unit % a.Hq), hk = h / (a.Hq / a.Hkv);
    if (t >= a.T || t >= a.cu[a.B]) return;
    int lo = 0, hi = a.B - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.cu[mid] <= t) lo = mid;
        else hi = mid - 1;
    }
    const int b = lo, i = t - a.cu[b], n_new = a.cu[b + 1] - a.cu[b];
    if (i < 0 || i >= n_new || i >= a.max_new) return;
    const int kv = (int)max(0LL, min((long long)a.kv_len[b], (long long)a.max_blocks * a.page));
    const int first = max(kv - n_new, 0);
    float q[kCh], o[kCh] = {}, m = -CUDART_INF_F, l = 0.0f;
#pragma unroll
    for (int e = 0; e < kCh; ++e) q[e] = __bfloat162float(a.q[t * a.q_t + h * a.q_h + lane * kCh + e]);
    const int last = a.mask_kind == DSP_MASK_CAUSAL ? min(kv, kv - n_new + i + 1) : kv;
    for (int u = 0; u < last; ++u) {
        if (a.mask_kind == DSP_MASK_BITS && u >= first) {
            const int j = u - (kv - n_new);
            if (j >= a.words * 32 || !((a.bits[(long long)t * a.words + (j >> 5)] >> (j & 31)) & 1u)) continue;
        }
        const int block = a.table[b * a.table_stride + u / a.page], place = u % a.page, tok = place & 15;
        if (block < 0 || block >= a.n_blocks) continue;
        const uint8_t *run = a.cache + run_index(block, place, hk, a.Hkv, a.page) * Kv4<D>::kRunBytes;
        const int word = lane * kCh / 8, c0 = lane * kCh % 8;
        const uint32_t kw = *reinterpret_cast<const uint32_t *>(run + Kv4<D>::key_word(tok, word));
        const uint32_t vw = *reinterpret_cast<const uint32_t *>(run + Kv4<D>::kValueOff + Kv4<D>::value_word(tok, word));
        const uint2 p = *reinterpret_cast<const uint2 *>(run + Kv4<D>::kParamOff + tok * 8);
        float s = 0.0f;
#pragma unroll
        for (int e = 0; e < kCh; ++e)
            s += q[e] * fmaf((float)((kw >> (4 * ((c0 + e) >> 1) + 16 * ((c0 + e) & 1))) & 15u), bf16_lo(p.x), bf16_hi(p.x));
#pragma unroll
        for (int x = 16; x > 0; x >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, x);
        s *= a.scale;
        if (s == -CUDART_INF_F) continue;
        const float top = fmaxf(m, s);
        const float w = __expf(s - top), keep = m == -CUDART_INF_F ? 0.0f : __expf(m - top);
        l = l * keep + w;
#pragma unroll
        for (int e = 0; e < kCh; ++e)
            o[e] = o[e] * keep + w * fmaf((float)((vw >> (4 * ((c0 + e) >> 1) + 16 * ((c0 + e) & 1))) & 15u), bf16_lo(p.y), bf16_hi(p.y));
        m = top;
    }
#pragma unroll
    for (int e = 0; e < kCh; ++e)
        a.out[((long long)t * a.Hq + h) * D + lane * kCh + e] = __float2bfloat16_rn(l == 0.0f ? 0.0f : o[e] / l);
}

}  // namespace
}  // namespace dsp

extern "C" int32_t dsp_attn_kv4_workspace_bytes(int32_t B, int32_t T, int32_t Hq, int32_t Hkv, int32_t D, int32_t max_new,
                                                size_t *bytes) {
    if (!bytes || B < 0 || T < 0 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0 || max_new < 1) return DSP_ERR_INVALID_ARG;
    if ((D != 64 && D != 128) || B > 65535 || T > (1 << 24) || Hq > 4096) return DSP_ERR_UNSUPPORTED;
    *bytes = 256;
    return DSP_OK;
}

extern "C" int32_t dsp_attn_kv4(const void *q, int32_t dtype, int32_t B, int32_t T, int32_t Hq, int32_t Hkv, int32_t D,
                                int64_t q_stride_t, int64_t q_stride_h,
                                const void *cache, int32_t n_blocks, int32_t page_size,
                                const int32_t *block_table, int64_t table_stride, int32_t max_blocks,
                                const int32_t *kv_len, const int32_t *cu_new, int32_t max_new, float scale,
                                int32_t mask_kind, const uint32_t *mask_bits, int32_t mask_words,
                                void *out, void *workspace, size_t workspace_bytes, dsp_stream_t stream) {
    using namespace dsp;
    size_t need = 0;
    const int32_t rc = dsp_attn_kv4_workspace_bytes(B, T, Hq, Hkv, D, max_new, &need);
    if (rc != DSP_OK) return rc;
    if (dtype != DSP_BF16) return DSP_ERR_UNSUPPORTED;
    if (n_blocks < 1 || page_size < 16 || page_size % 16 != 0 || max_blocks < 1 || table_stride < max_blocks) return DSP_ERR_INVALID_ARG;
    if (!isfinite(scale)) return DSP_ERR_INVALID_ARG;
    if (mask_kind != DSP_MASK_CAUSAL && mask_kind != DSP_MASK_FULL && mask_kind != DSP_MASK_BITS) return DSP_ERR_INVALID_ARG;
    if (B == 0 || T == 0) return DSP_OK;
    if (!q || !cache || !block_table || !kv_len || !cu_new || !out || !workspace) return DSP_ERR_INVALID_ARG;
    if ((mask_kind == DSP_MASK_BITS) != (mask_bits != nullptr) || (mask_bits && mask_words < 1)) return DSP_ERR_INVALID_ARG;
    if (q_stride_h < D || q_stride_t < (int64_t)(Hq - 1) * q_stride_h + D) return DSP_ERR_INVALID_ARG;
    const uintptr_t all16 = reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out) | reinterpret_cast<uintptr_t>(cache);
    if ((all16 & 15) || q_stride_t % 8 || q_stride_h % 8 || (reinterpret_cast<uintptr_t>(workspace) & 255)) return DSP_ERR_INVALID_ARG;
    if (workspace_bytes < need) return DSP_ERR_WORKSPACE;
    AttnArgs a = {};
    a.q = static_cast<const __nv_bfloat16 *>(q);
    a.q_t = q_stride_t; a.q_h = q_stride_h;
    a.B = B; a.T = T; a.Hq = Hq; a.Hkv = Hkv;
    a.cache = static_cast<const uint8_t *>(cache); a.n_blocks = n_blocks; a.page = page_size;
    a.table = block_table; a.table_stride = table_stride; a.max_blocks = max_blocks;
    a.kv_len = kv_len; a.cu = cu_new; a.max_new = max_new;
    a.scale = scale; a.mask_kind = mask_kind; a.bits = mask_bits; a.words = mask_words;
    a.out = static_cast<__nv_bfloat16 *>(out);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const long long units = (long long)T * Hq;
    const unsigned grid = (unsigned)((units + 3) / 4);
    if (D == 64) attn_simple_kernel<64><<<grid, 128, 0, st>>>(a);
    else attn_simple_kernel<128><<<grid, 128, 0, st>>>(a);
    DSP_CUDA_TRY(cudaGetLastError());
    return DSP_OK;
}
