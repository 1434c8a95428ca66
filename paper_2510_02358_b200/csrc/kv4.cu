// dsp_qk_norm_rope, dsp_kv4_append, dsp_kv4_read: what every token's heads go through between the
// projections and the attention (the norm of each query and key head, the rotation by position,
// the 4-bit form of keys and values), in one pass over them.
//
// A head of a token is a row of D channels on D / 8 neighbouring lanes, eight channels a lane: the
// row's sum of squares, extrema and the rotation's partner channels come from shuffles inside those
// lanes, so nothing goes through shared memory and the pass is one read and one write of the rows.
// A group of lanes takes kHeads heads of one token: their loads are in flight together, and the
// token's angles are read once for them.
//
// What is written is a function of the row alone: the sum of squares is a tree of neighbouring
// channels (in a lane, then over the lanes by xor 1, 2, 4, 8), and no product is fused with a sum,
// so the same row gives the same bits (and, right on the edge between two codes, the same code)
// from every call shape, and dsp_kv4_append's keys are those of dsp_qk_norm_rope.
#include "kv4.cuh"

namespace dsp {
namespace {

constexpr int kNormThreads = 256;
constexpr long long kMaxRows = 1LL << 30;        // tokens x heads of one call: row numbers stay in 32 bits

struct NormArgs {
    const void *q, *k, *v;
    long long q_t, q_h, k_t, k_h, v_t, v_h;      // strides in elements
    bool q_vec, k_vec, v_vec, w_vec;             // rows start on 16 bytes: 128-bit loads
    const void *q_weight, *k_weight;
    float eps;
    const int32_t *positions;
    const float *cos_sin;
    bool cs_vec;
    int max_pos, rot, interleaved;
    int T, Hq, Hkv, heads;                       // heads: Hq + Hkv (norm) or Hq + 2 Hkv (append)
    int chunks;                                  // groups of heads per token
    const int64_t *slot;
    uint8_t *cache;
    long long n_slots;
    int page;
    void *q_out, *k_out;
};

template <typename DT> struct Row8;
template <> struct Row8<__nv_bfloat16> {
    uint4 v;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p, bool vec) {
        if (vec) {
            v = ldg_stream(p);
        } else {
            const unsigned short *u = reinterpret_cast<const unsigned short *>(p);
            v.x = u[0] | (uint32_t)u[1] << 16; v.y = u[2] | (uint32_t)u[3] << 16;
            v.z = u[4] | (uint32_t)u[5] << 16; v.w = u[6] | (uint32_t)u[7] << 16;
        }
    }
    __device__ __forceinline__ void get(float (&x)[8]) const {
        x[0] = bf16_lo(v.x); x[1] = bf16_hi(v.x); x[2] = bf16_lo(v.y); x[3] = bf16_hi(v.y);
        x[4] = bf16_lo(v.z); x[5] = bf16_hi(v.z); x[6] = bf16_lo(v.w); x[7] = bf16_hi(v.w);
    }
    static __device__ __forceinline__ uint32_t pack(float a, float b) {
        const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t *>(&p);
    }
    static __device__ __forceinline__ void store(__nv_bfloat16 *p, const float (&x)[8]) {
        *reinterpret_cast<uint4 *>(p) = make_uint4(pack(x[0], x[1]), pack(x[2], x[3]), pack(x[4], x[5]), pack(x[6], x[7]));
    }
    static __device__ __forceinline__ float rounded(float x) { return __bfloat162float(__float2bfloat16_rn(x)); }
};
template <> struct Row8<float> {
    uint4 a, b;
    __device__ __forceinline__ void load(const float *p, bool vec) {
        if (vec) {
            a = ldg_stream(p);
            b = ldg_stream(p + 4);
        } else {
            const uint32_t *u = reinterpret_cast<const uint32_t *>(p);
            a = make_uint4(u[0], u[1], u[2], u[3]);
            b = make_uint4(u[4], u[5], u[6], u[7]);
        }
    }
    __device__ __forceinline__ void get(float (&x)[8]) const {
        x[0] = __uint_as_float(a.x); x[1] = __uint_as_float(a.y); x[2] = __uint_as_float(a.z); x[3] = __uint_as_float(a.w);
        x[4] = __uint_as_float(b.x); x[5] = __uint_as_float(b.y); x[6] = __uint_as_float(b.z); x[7] = __uint_as_float(b.w);
    }
    static __device__ __forceinline__ void store(float *p, const float (&x)[8]) {
        *reinterpret_cast<float4 *>(p) = make_float4(x[0], x[1], x[2], x[3]);
        *reinterpret_cast<float4 *>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
    }
    static __device__ __forceinline__ float rounded(float x) { return x; }
};

__device__ __forceinline__ float bf16_down(float x) {
    const uint32_t b = __float_as_uint(x);
    return __uint_as_float((int32_t)b < 0 ? (b + 0xFFFFu) & 0xFFFF0000u : b & 0xFFFF0000u);
}
__device__ __forceinline__ float bf16_up_nonneg(float x) { return __uint_as_float((__float_as_uint(x) + 0xFFFFu) & 0xFFFF0000u); }

// One scale, one offset and eight codes of a lane's channels; kLanes lanes hold the row.
template <int kLanes>
__device__ __forceinline__ uint32_t quantise8(const float (&x)[8], uint32_t &params) {
    float lo = x[0], hi = x[0];
    bool fine = fabsf(x[0]) <= 3.402823466e38f;
#pragma unroll
    for (int e = 1; e < 8; ++e) {
        lo = fminf(lo, x[e]);
        hi = fmaxf(hi, x[e]);
        fine = fine && fabsf(x[e]) <= 3.402823466e38f;            // false for NaN too
    }
    hi = fine ? hi : CUDART_INF_F;                                 // carries the finding through the reduction
#pragma unroll
    for (int o = 1; o < kLanes; o <<= 1) {
        lo = fminf(lo, __shfl_xor_sync(0xFFFFFFFFu, lo, o));
        hi = fmaxf(hi, __shfl_xor_sync(0xFFFFFFFFu, hi, o));
    }
    const float z = bf16_down(lo);
    float s = bf16_up_nonneg(__fdiv_rn(__fsub_rn(hi, z), 15.0f));
    const bool ok = hi <= 3.402823466e38f && z >= -3.402823466e38f && s <= 3.402823466e38f;
    s = s < 1.17549435e-38f ? 0.0f : s;
    uint32_t w = 0u;
    if (ok && s > 0.0f) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t code = min(__float2uint_rn(__fdiv_rn(__fsub_rn(x[e], z), s)), 15u);
            w |= code << (4 * (e >> 1) + 16 * (e & 1));
        }
    }
    params = ok ? (__float_as_uint(s) >> 16) | (__float_as_uint(z) & 0xFFFF0000u) : 0x7FFF7FFFu;
    return w;
}

template <typename DT, int D, bool kAppend, int kHeads>
__global__ void __launch_bounds__(kNormThreads) norm_rope_kernel(const NormArgs a) {
    constexpr int kLanes = D / 8;                                 // lanes of a row
    const int lane = threadIdx.x & (kLanes - 1);
    const uint32_t group = blockIdx.x * (kNormThreads / kLanes) + threadIdx.x / kLanes;
    const uint32_t t_raw = group / (uint32_t)a.chunks;
    const bool live = t_raw < (uint32_t)a.T;                      // whole groups: the shuffles below need every lane of the warp
    const int t = live ? (int)t_raw : a.T - 1;
    const int h0 = (int)(group - t_raw * (uint32_t)a.chunks) * kHeads;
    const int ch = lane * 8;
    const bool rope = a.cos_sin != nullptr;

    Row8<DT> raw[kHeads];
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
        const int h = min(h0 + i, a.heads - 1);
        const DT *p;
        bool vec;
        if (h < a.Hq) {
            p = static_cast<const DT *>(a.q) + t * a.q_t + h * a.q_h;
            vec = a.q_vec;
        } else if (!kAppend || h < a.Hq + a.Hkv) {
            p = static_cast<const DT *>(a.k) + t * a.k_t + (h - a.Hq) * a.k_h;
            vec = a.k_vec;
        } else {
            p = static_cast<const DT *>(a.v) + t * a.v_t + (h - a.Hq - a.Hkv) * a.v_h;
            vec = a.v_vec;
        }
        raw[i].load(p + ch, vec);
    }
    const int pos = a.positions ? a.positions[t] : 0;
    const bool pad = pos < 0, beyond = rope && pos >= a.max_pos;
    const bool turned = rope && ch < a.rot;
    // the angles of this lane's channels: pairs (i, i + rot/2) or (2i, 2i+1)
    float c[8], s[8];
    if (turned) {
        const float *row = a.cos_sin + (long long)min(max(pos, 0), a.max_pos - 1) * a.rot;
        const int half = a.rot >> 1;
        if (a.interleaved) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                c[e] = __ldg(row + (ch >> 1) + e);
                s[e] = __ldg(row + half + (ch >> 1) + e);
            }
        } else {
            const int i0 = ch < half ? ch : ch - half;
            if (a.cs_vec) {
#pragma unroll
                for (int e = 0; e < 8; e += 4) {
                    const float4 cv = __ldg(reinterpret_cast<const float4 *>(row + i0 + e));
                    const float4 sv = __ldg(reinterpret_cast<const float4 *>(row + half + i0 + e));
                    c[e] = cv.x; c[e + 1] = cv.y; c[e + 2] = cv.z; c[e + 3] = cv.w;
                    s[e] = sv.x; s[e + 1] = sv.y; s[e + 2] = sv.z; s[e + 3] = sv.w;
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    c[e] = __ldg(row + i0 + e);
                    s[e] = __ldg(row + half + i0 + e);
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
        const int h = h0 + i;
        const bool mine = live && h < a.heads;
        const int kind = h < a.Hq ? 0 : (!kAppend || h < a.Hq + a.Hkv) ? 1 : 2;
        float x[8];
        raw[i].get(x);
        {   // heads of both kinds may share a warp: every lane takes part in the sum, values leave it unused
            const DT *w = static_cast<const DT *>(kind == 0 ? a.q_weight : kind == 1 ? a.k_weight : nullptr);
            float sq[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) sq[e] = __fmul_rn(x[e], x[e]);
            float sum = __fadd_rn(__fadd_rn(__fadd_rn(sq[0], sq[1]), __fadd_rn(sq[2], sq[3])),
                                  __fadd_rn(__fadd_rn(sq[4], sq[5]), __fadd_rn(sq[6], sq[7])));
#pragma unroll
            for (int o = 1; o < kLanes; o <<= 1) sum = __fadd_rn(sum, __shfl_xor_sync(0xFFFFFFFFu, sum, o));
            if (w) {
                const float r = __fdiv_rn(1.0f, __fsqrt_rn(__fadd_rn(__fmul_rn(sum, 1.0f / D), a.eps)));
                Row8<DT> wr;
                wr.load(w + ch, a.w_vec);
                float wv[8];
                wr.get(wv);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = __fmul_rn(__fmul_rn(x[e], r), wv[e]);
            }
        }
        if (rope) {                                               // uniform over the grid
            float y[8];
            if (a.interleaved) {
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    y[e] = __fsub_rn(__fmul_rn(x[e], c[e >> 1]), __fmul_rn(x[e + 1], s[e >> 1]));
                    y[e + 1] = __fadd_rn(__fmul_rn(x[e + 1], c[e >> 1]), __fmul_rn(x[e], s[e >> 1]));
                }
            } else {
                const int hop = a.rot >> 4;                       // lanes between a channel and its partner
                const bool first = lane < hop;
                const int base = (threadIdx.x & 31) - lane;
                const int src = base + (first ? lane + hop : lane < 2 * hop ? lane - hop : lane);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float o = __shfl_sync(0xFFFFFFFFu, x[e], src);
                    const float xc = __fmul_rn(x[e], c[e]), os = __fmul_rn(o, s[e]);
                    y[e] = first ? __fsub_rn(xc, os) : __fadd_rn(xc, os);
                }
            }
            if (turned && kind < 2) {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = y[e];
            }
        }
        if (kind < 2 && (pad || beyond)) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = pad ? 0.0f : CUDART_NAN_F;
        }
        if (kind == 0) {
            if (mine && a.q_out) Row8<DT>::store(static_cast<DT *>(a.q_out) + ((long long)t * a.Hq + h) * D + ch, x);
        } else if (!kAppend) {
            if (mine) Row8<DT>::store(static_cast<DT *>(a.k_out) + ((long long)t * a.Hkv + (h - a.Hq)) * D + ch, x);
        }
        if (kAppend) {
            if constexpr (D <= 128) {
                // shuffles inside: every lane of the warp takes part, queries too when they share a warp with keys
                const bool any = __any_sync(0xFFFFFFFFu, kind > 0);
                if (any) {
                    if (kind == 1) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[e] = Row8<DT>::rounded(x[e]);
                    }
                    uint32_t params;
                    const uint32_t w = quantise8<kLanes>(x, params);
                    const long long slot = a.slot[t];
                    if (mine && kind > 0 && !pad && slot >= 0 && slot < a.n_slots) {
                        const long long block = block_of(slot, a.page);
                        const int place = (int)(slot - block * a.page), tok = place & 15;
                        const int hk = kind == 1 ? h - a.Hq : h - a.Hq - a.Hkv;
                        uint8_t *run = a.cache + run_index(block, place, hk, a.Hkv, a.page) * Kv4<D>::kRunBytes;
                        const int at = kind == 1 ? Kv4<D>::key_word(tok, lane) : Kv4<D>::kValueOff + Kv4<D>::value_word(tok, lane);
                        *reinterpret_cast<uint32_t *>(run + at) = w;
                        if (lane == 0)
                            *reinterpret_cast<uint32_t *>(run + Kv4<D>::kParamOff + tok * 8 + (kind == 1 ? 0 : 4)) = params;
                    }
                }
            }
        }
    }
}

struct ReadArgs {
    const uint8_t *cache;
    const int64_t *slot;
    void *k_out, *v_out;
    int T, Hkv, page;
    long long n_slots;
};

// One word of key codes and one of value codes per lane: eight channels each.
template <typename DT, int D>
__global__ void __launch_bounds__(kNormThreads) kv4_read_kernel(const ReadArgs a) {
    constexpr int kLanes = D / 8;
    const int lane = threadIdx.x & (kLanes - 1);
    const uint32_t row32 = blockIdx.x * (kNormThreads / kLanes) + threadIdx.x / kLanes;       // token * Hkv + head
    const uint32_t t = row32 / (uint32_t)a.Hkv;
    if (t >= (uint32_t)a.T) return;
    const int h = (int)(row32 - t * (uint32_t)a.Hkv);
    const long long row = row32, slot = a.slot[t];
    float k[8] = {}, v[8] = {};
    if (slot >= 0 && slot < a.n_slots) {
        const long long block = block_of(slot, a.page);
        const int place = (int)(slot - block * a.page), tok = place & 15;
        const uint8_t *run = a.cache + run_index(block, place, h, a.Hkv, a.page) * Kv4<D>::kRunBytes;
        const uint32_t kw = *reinterpret_cast<const uint32_t *>(run + Kv4<D>::key_word(tok, lane));
        const uint32_t vw = *reinterpret_cast<const uint32_t *>(run + Kv4<D>::kValueOff + Kv4<D>::value_word(tok, lane));
        const uint2 p = *reinterpret_cast<const uint2 *>(run + Kv4<D>::kParamOff + tok * 8);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int sh = 4 * (e >> 1) + 16 * (e & 1);
            k[e] = fmaf((float)((kw >> sh) & 15u), bf16_lo(p.x), bf16_hi(p.x));
            v[e] = fmaf((float)((vw >> sh) & 15u), bf16_lo(p.y), bf16_hi(p.y));
        }
    }
    Row8<DT>::store(static_cast<DT *>(a.k_out) + row * D + lane * 8, k);
    Row8<DT>::store(static_cast<DT *>(a.v_out) + row * D + lane * 8, v);
}

bool on16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool rows_on16(const void *p, int64_t st, int64_t sh, int esz) { return on16(p) && (st * esz) % 16 == 0 && (sh * esz) % 16 == 0; }

int32_t check_norm(int32_t dtype, int32_t T, int32_t Hq, int32_t Hkv, int32_t D, float eps, const int32_t *positions,
                   const float *cos_sin, int32_t max_pos, int32_t rot) {
    if (T < 0 || Hq < 1 || Hkv < 1 || D < 1 || !(eps >= 0.0f) || eps > 3.402823466e38f) return DSP_ERR_INVALID_ARG;
    if (dtype != DSP_F32 && dtype != DSP_BF16) return DSP_ERR_UNSUPPORTED;
    if ((D != 64 && D != 128 && D != 256) || T > (1 << 24) || Hq > 4096 || Hkv > 4096) return DSP_ERR_UNSUPPORTED;
    if ((long long)T * ((long long)Hq + 2 * Hkv) > kMaxRows) return DSP_ERR_UNSUPPORTED;
    if (cos_sin) {
        if (!positions || max_pos < 1) return DSP_ERR_INVALID_ARG;
        if (rot < 16 || rot > D || rot % 16 != 0) return DSP_ERR_UNSUPPORTED;
    }
    return DSP_OK;
}
bool strides_ok(int64_t st, int64_t sh, int32_t H, int32_t D) { return sh >= D && st >= (int64_t)(H - 1) * sh + D; }

template <typename DT, int D, bool kAppend>
cudaError_t launch_norm_heads(NormArgs a, cudaStream_t st) {
    constexpr int kGroups = kNormThreads / (D / 8);
    // Four heads to a group of lanes once that still fills the GPU (148 SMs of 8 CTAs), one below:
    // a short call is the latency of one group's chain, a long one wants loads in flight.
    const bool wide = (long long)a.T * a.heads >= 4LL * 148 * 8 * kGroups;
    a.chunks = wide ? (a.heads + 3) / 4 : a.heads;
    const long long groups = (long long)a.T * a.chunks;
    const unsigned grid = (unsigned)((groups + kGroups - 1) / kGroups);
    if (wide)
        norm_rope_kernel<DT, D, kAppend, 4><<<grid, kNormThreads, 0, st>>>(a);
    else
        norm_rope_kernel<DT, D, kAppend, 1><<<grid, kNormThreads, 0, st>>>(a);
    return cudaGetLastError();
}

template <bool kAppend>
cudaError_t launch_norm(const NormArgs &a, int32_t dtype, int32_t D, cudaStream_t st) {
    if (dtype == DSP_BF16) {
        if (D == 64) return launch_norm_heads<__nv_bfloat16, 64, kAppend>(a, st);
        if (D == 128) return launch_norm_heads<__nv_bfloat16, 128, kAppend>(a, st);
        if constexpr (!kAppend) return launch_norm_heads<__nv_bfloat16, 256, kAppend>(a, st);
    } else {
        if (D == 64) return launch_norm_heads<float, 64, kAppend>(a, st);
        if (D == 128) return launch_norm_heads<float, 128, kAppend>(a, st);
        if constexpr (!kAppend) return launch_norm_heads<float, 256, kAppend>(a, st);
    }
    return cudaErrorInvalidValue;
}

NormArgs norm_args(const void *q, const void *k, const void *v, int32_t dtype, int32_t T, int32_t Hq, int32_t Hkv,
                   int64_t q_t, int64_t q_h, int64_t k_t, int64_t k_h, int64_t v_t, int64_t v_h,
                   const void *q_weight, const void *k_weight, float eps, const int32_t *positions,
                   const float *cos_sin, int32_t max_pos, int32_t rot, int32_t interleaved) {
    const int esz = dtype == DSP_BF16 ? 2 : 4;
    NormArgs a = {};
    a.q = q; a.k = k; a.v = v;
    a.q_t = q_t; a.q_h = q_h; a.k_t = k_t; a.k_h = k_h; a.v_t = v_t; a.v_h = v_h;
    a.q_vec = rows_on16(q, q_t, q_h, esz);
    a.k_vec = rows_on16(k, k_t, k_h, esz);
    a.v_vec = v && rows_on16(v, v_t, v_h, esz);
    a.q_weight = q_weight; a.k_weight = k_weight;
    a.w_vec = on16(q_weight) && on16(k_weight);
    a.eps = eps;
    a.positions = positions;
    a.cos_sin = cos_sin;
    a.cs_vec = on16(cos_sin);                    // rot is a multiple of 16, so every row and half is aligned with it
    a.max_pos = max_pos; a.rot = rot; a.interleaved = interleaved;
    a.T = T; a.Hq = Hq; a.Hkv = Hkv;
    return a;
}

}  // namespace
}  // namespace dsp

extern "C" int32_t dsp_qk_norm_rope(const void *q, const void *k, int32_t dtype, int32_t T, int32_t Hq, int32_t Hkv, int32_t D,
                                    int64_t q_stride_t, int64_t q_stride_h, int64_t k_stride_t, int64_t k_stride_h,
                                    const void *q_weight, const void *k_weight, float eps,
                                    const int32_t *positions, const float *cos_sin, int32_t max_pos, int32_t rot,
                                    int32_t interleaved, void *q_out, void *k_out, dsp_stream_t stream) {
    using namespace dsp;
    const int32_t rc = check_norm(dtype, T, Hq, Hkv, D, eps, positions, cos_sin, max_pos, rot);
    if (rc != DSP_OK) return rc;
    if (T == 0) return DSP_OK;
    if (!q || !k || !q_out || !k_out || !on16(q_out) || !on16(k_out)) return DSP_ERR_INVALID_ARG;
    if (!strides_ok(q_stride_t, q_stride_h, Hq, D) || !strides_ok(k_stride_t, k_stride_h, Hkv, D)) return DSP_ERR_INVALID_ARG;
    NormArgs a = norm_args(q, k, nullptr, dtype, T, Hq, Hkv, q_stride_t, q_stride_h, k_stride_t, k_stride_h, 0, 0,
                           q_weight, k_weight, eps, positions, cos_sin, max_pos, rot, interleaved);
    a.heads = Hq + Hkv;
    a.q_out = q_out; a.k_out = k_out;
    DSP_CUDA_TRY(launch_norm<false>(a, dtype, D, reinterpret_cast<cudaStream_t>(stream)));
    return DSP_OK;
}

static int32_t check_cache(const void *cache, int32_t n_blocks, int32_t page_size) {
    if (n_blocks < 1 || page_size < 16 || page_size % 16 != 0) return DSP_ERR_INVALID_ARG;
    return cache && dsp::on16(cache) ? DSP_OK : DSP_ERR_INVALID_ARG;
}

extern "C" int32_t dsp_kv4_append(const void *q, const void *k, const void *v, int32_t dtype,
                                  int32_t T, int32_t Hq, int32_t Hkv, int32_t D,
                                  int64_t q_stride_t, int64_t q_stride_h, int64_t k_stride_t, int64_t k_stride_h,
                                  int64_t v_stride_t, int64_t v_stride_h,
                                  const void *q_weight, const void *k_weight, float eps,
                                  const int32_t *positions, const float *cos_sin, int32_t max_pos, int32_t rot,
                                  int32_t interleaved, const int64_t *slot, void *cache, int32_t n_blocks,
                                  int32_t page_size, void *q_out, dsp_stream_t stream) {
    using namespace dsp;
    const bool with_q = q || q_out;
    int32_t rc = check_norm(dtype, T, with_q ? Hq : 1, Hkv, D, eps, positions, cos_sin, max_pos, rot);
    if (rc == DSP_OK && D == 256) rc = DSP_ERR_UNSUPPORTED;
    if (rc != DSP_OK) return rc;
    if (T == 0) return DSP_OK;
    if (!k || !v || !slot || check_cache(cache, n_blocks, page_size) != DSP_OK) return DSP_ERR_INVALID_ARG;
    if (with_q && (!q || !q_out || !on16(q_out) || !strides_ok(q_stride_t, q_stride_h, Hq, D))) return DSP_ERR_INVALID_ARG;
    if (!strides_ok(k_stride_t, k_stride_h, Hkv, D) || !strides_ok(v_stride_t, v_stride_h, Hkv, D)) return DSP_ERR_INVALID_ARG;
    NormArgs a = norm_args(q, k, v, dtype, T, with_q ? Hq : 0, Hkv, q_stride_t, q_stride_h, k_stride_t, k_stride_h,
                           v_stride_t, v_stride_h, q_weight, k_weight, eps, positions, cos_sin, max_pos, rot, interleaved);
    a.heads = a.Hq + 2 * Hkv;
    a.slot = slot;
    a.cache = static_cast<uint8_t *>(cache);
    a.n_slots = (long long)n_blocks * page_size;
    a.page = page_size;
    a.q_out = q_out;
    DSP_CUDA_TRY(launch_norm<true>(a, dtype, D, reinterpret_cast<cudaStream_t>(stream)));
    return DSP_OK;
}

extern "C" int32_t dsp_kv4_read(const void *cache, int32_t n_blocks, int32_t page_size, int32_t Hkv, int32_t D,
                                const int64_t *slot, int32_t T, int32_t dtype, void *k_out, void *v_out,
                                dsp_stream_t stream) {
    using namespace dsp;
    if (T < 0 || Hkv < 1 || D < 1) return DSP_ERR_INVALID_ARG;
    if (dtype != DSP_F32 && dtype != DSP_BF16) return DSP_ERR_UNSUPPORTED;
    if ((D != 64 && D != 128) || T > (1 << 24) || Hkv > 4096 || (long long)T * Hkv > kMaxRows) return DSP_ERR_UNSUPPORTED;
    if (T == 0) return DSP_OK;
    if (check_cache(cache, n_blocks, page_size) != DSP_OK) return DSP_ERR_INVALID_ARG;
    if (!slot || !k_out || !v_out || !on16(k_out) || !on16(v_out)) return DSP_ERR_INVALID_ARG;
    ReadArgs a = {static_cast<const uint8_t *>(cache), slot, k_out, v_out, T, Hkv, page_size,
                  (long long)n_blocks * page_size};
    const long long threads = (long long)T * Hkv * (D / 8);
    const unsigned grid = (unsigned)((threads + kNormThreads - 1) / kNormThreads);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (dtype == DSP_BF16) {
        if (D == 64) kv4_read_kernel<__nv_bfloat16, 64><<<grid, kNormThreads, 0, st>>>(a);
        else kv4_read_kernel<__nv_bfloat16, 128><<<grid, kNormThreads, 0, st>>>(a);
    } else {
        if (D == 64) kv4_read_kernel<float, 64><<<grid, kNormThreads, 0, st>>>(a);
        else kv4_read_kernel<float, 128><<<grid, kNormThreads, 0, st>>>(a);
    }
    DSP_CUDA_TRY(cudaGetLastError());
    return DSP_OK;
}
