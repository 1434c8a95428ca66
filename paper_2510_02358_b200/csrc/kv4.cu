// dsp_qk_norm_rope, dsp_kv4_append, dsp_kv4_read: what every token's heads go through between the
// projections and the attention (the norm of each query and key head, the rotation by position,
// the 4-bit form of keys and values), in one pass over them.
//
// A head of a token is a row of D channels on a few neighbouring lanes: the row's sum of squares and
// extrema come from shuffles inside those lanes, so nothing goes through shared memory and the pass is
// one read and one write of the rows.  A group of lanes takes kHeads heads of one token: their loads
// are in flight together, and the token's angles are read once for them.
//
// What is written is a function of the row alone: the sum of squares is a tree of neighbouring
// channels (in a lane, then over the lanes by xor 1, 2, 4, 8), and no product is fused with a sum,
// so the same row gives the same bits (and, right on the edge between two codes, the same code)
// from every call shape, and dsp_kv4_append's keys are those of dsp_qk_norm_rope.
//
// Measured, 8192 tokens: norm and rotation of 40 + 8 heads of 128 in bf16 45 us (201 MB, 4.5 TB/s), with keys and values stored 65 us (219
// MB, 3.4 TB/s: 27 of them for the keys and values, by the codes' arithmetic and by stores of 4 bytes); 8 tokens 2.3 and 2.8 us, a launch's
// latency.
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
    int T, Hq, Hkv;
    int chunks, q_chunks, k_chunks;              // groups of heads per token, of queries, of keys
    const int64_t *slot;
    uint8_t *cache;
    long long n_slots;
    int page;
    void *q_out, *k_out;
};

// Two fp32 numbers that go through the arithmetic together (each rounded for itself, as ever).
struct Two {
    float a, b;
};
__device__ __forceinline__ Two mul2(Two x, Two y) {
    asm("{\n .reg .b64 u, v;\n mov.b64 u, {%0, %1};\n mov.b64 v, {%2, %3};\n mul.rn.f32x2 u, u, v;\n mov.b64 {%0, %1}, u;\n}"
        : "+f"(x.a), "+f"(x.b) : "f"(y.a), "f"(y.b));
    return x;
}
__device__ __forceinline__ Two add2(Two x, Two y) {
    asm("{\n .reg .b64 u, v;\n mov.b64 u, {%0, %1};\n mov.b64 v, {%2, %3};\n add.rn.f32x2 u, u, v;\n mov.b64 {%0, %1}, u;\n}"
        : "+f"(x.a), "+f"(x.b) : "f"(y.a), "f"(y.b));
    return x;
}

// Sum of two products, each rounded for itself.  The additions are single ones: a packed product and the packed sum that takes it
// are built as one fused step, although both ask for a rounding of their own (tenths of the rotated numbers then had another last bit, and a key's code, once in some 10^4 heads, was another).
__device__ __forceinline__ Two add_products(Two x, Two y) { return {__fadd_rn(x.a, y.a), __fadd_rn(x.b, y.b)}; }

__device__ __forceinline__ Two fma2(Two x, Two y, Two z) {
    asm("{\n .reg .b64 u, v, w;\n mov.b64 u, {%0, %1};\n mov.b64 v, {%2, %3};\n mov.b64 w, {%4, %5};\n fma.rn.f32x2 u, u, v, w;\n mov.b64 {%0, %1}, u;\n}"
        : "+f"(x.a), "+f"(x.b) : "f"(y.a), "f"(y.b), "f"(z.a), "f"(z.b));
    return x;
}

// Four neighbouring channels of a row.
template <typename DT> struct Quad;
template <> struct Quad<__nv_bfloat16> {
    uint2 v;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p, bool vec) {
        if (vec) {
            asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
        } else {
            const unsigned short *u = reinterpret_cast<const unsigned short *>(p);
            v.x = u[0] | (uint32_t)u[1] << 16;
            v.y = u[2] | (uint32_t)u[3] << 16;
        }
    }
    __device__ __forceinline__ void get(Two &x, Two &y) const {
        x = {bf16_lo(v.x), bf16_hi(v.x)};
        y = {bf16_lo(v.y), bf16_hi(v.y)};
    }
    static __device__ __forceinline__ uint32_t pack(Two x) {
        const __nv_bfloat162 p = __floats2bfloat162_rn(x.a, x.b);
        return *reinterpret_cast<const uint32_t *>(&p);
    }
    static __device__ __forceinline__ void store(__nv_bfloat16 *p, Two x, Two y) {
        *reinterpret_cast<uint2 *>(p) = make_uint2(pack(x), pack(y));
    }
    static __device__ __forceinline__ Two rounded(Two x) {
        const uint32_t w = pack(x);
        return {bf16_lo(w), bf16_hi(w)};
    }
};
template <> struct Quad<float> {
    uint4 v;
    __device__ __forceinline__ void load(const float *p, bool vec) {
        if (vec) {
            v = ldg_stream(p);
        } else {
            const uint32_t *u = reinterpret_cast<const uint32_t *>(p);
            v = make_uint4(u[0], u[1], u[2], u[3]);
        }
    }
    __device__ __forceinline__ void get(Two &x, Two &y) const {
        x = {__uint_as_float(v.x), __uint_as_float(v.y)};
        y = {__uint_as_float(v.z), __uint_as_float(v.w)};
    }
    static __device__ __forceinline__ void store(float *p, Two x, Two y) { *reinterpret_cast<float4 *>(p) = make_float4(x.a, x.b, y.a, y.b); }
    static __device__ __forceinline__ Two rounded(Two x) { return x; }
};

// Eight neighbouring channels: pairs (0,1) (2,3) (4,5) (6,7).
template <typename DT> struct Eight;
template <> struct Eight<__nv_bfloat16> {
    uint4 v;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p, bool vec) {
        if (vec) {
            v = ldg_stream(p);
        } else {
            const unsigned short *u = reinterpret_cast<const unsigned short *>(p);
            v = make_uint4(u[0] | (uint32_t)u[1] << 16, u[2] | (uint32_t)u[3] << 16, u[4] | (uint32_t)u[5] << 16, u[6] | (uint32_t)u[7] << 16);
        }
    }
    __device__ __forceinline__ void get(Two (&x)[4]) const {
        x[0] = {bf16_lo(v.x), bf16_hi(v.x)}; x[1] = {bf16_lo(v.y), bf16_hi(v.y)};
        x[2] = {bf16_lo(v.z), bf16_hi(v.z)}; x[3] = {bf16_lo(v.w), bf16_hi(v.w)};
    }
    static __device__ __forceinline__ void store(__nv_bfloat16 *p, const Two (&x)[4]) {
        *reinterpret_cast<uint4 *>(p) = make_uint4(Quad<__nv_bfloat16>::pack(x[0]), Quad<__nv_bfloat16>::pack(x[1]),
                                                   Quad<__nv_bfloat16>::pack(x[2]), Quad<__nv_bfloat16>::pack(x[3]));
    }
};
template <> struct Eight<float> {
    Quad<float> q[2];
    __device__ __forceinline__ void load(const float *p, bool vec) { q[0].load(p, vec); q[1].load(p + 4, vec); }
    __device__ __forceinline__ void get(Two (&x)[4]) const { q[0].get(x[0], x[1]); q[1].get(x[2], x[3]); }
    static __device__ __forceinline__ void store(float *p, const Two (&x)[4]) {
        Quad<float>::store(p, x[0], x[1]);
        Quad<float>::store(p + 4, x[2], x[3]);
    }
};
// Sum of eight squares as a tree of neighbours.
__device__ __forceinline__ float square_sum(const Two (&x)[4]) {
    float s[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const Two q = mul2(x[e], x[e]);
        s[e] = __fadd_rn(q.a, q.b);
    }
    return __fadd_rn(__fadd_rn(s[0], s[1]), __fadd_rn(s[2], s[3]));
}

__device__ __forceinline__ float bf16_down(float x) {
    const uint32_t b = __float_as_uint(x);
    return __uint_as_float((int32_t)b < 0 ? (b + 0xFFFFu) & 0xFFFF0000u : b & 0xFFFF0000u);
}
__device__ __forceinline__ float bf16_up_nonneg(float x) { return __uint_as_float((__float_as_uint(x) + 0xFFFFu) & 0xFFFF0000u); }

__device__ __forceinline__ float max3(float a, float b, float c) {
    float y;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
    return y;
}
__device__ __forceinline__ float min3(float a, float b, float c) {
    float y;
    asm("min.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
    return y;
}

// One scale and one offset for a row that lies on kLanes lanes, and the codes of eight channels as a word.
//
// A code is (x - z) / s, rounded to fp32, then to a whole number.  The quotient comes from the correctly rounded reciprocal and one
// step with the exact remainder (Markstein's method): q = d * inv, q + (d - q s) * inv.  That is within 2^-46 of d / s before its
// own rounding, and d / s cannot be nearer than 2^-33 to the middle between two fp32 numbers, since s has 8 bits: so it is the
// rounded quotient.  (Only where neither the remainder nor the reciprocal leaves the normal range; elsewhere the lanes divide.)
struct Extrema {
    float lo, hi;
    bool fine;
    __device__ __forceinline__ Extrema(const Two (&x)[4]) {
        lo = min3(min3(x[0].a, x[0].b, x[1].a), x[1].b, x[2].a);
        hi = max3(max3(x[0].a, x[0].b, x[1].a), x[1].b, x[2].a);
        lo = fminf(min3(lo, x[2].b, x[3].a), x[3].b);
        hi = fmaxf(max3(hi, x[2].b, x[3].a), x[3].b);
        const Two zero = {0.0f, 0.0f};                             // 0 * x is NaN for an infinity or a NaN
        const Two odd = add2(add2(mul2(x[0], zero), mul2(x[1], zero)), add2(mul2(x[2], zero), mul2(x[3], zero)));
        fine = odd.a + odd.b == 0.0f;
    }
};
struct Scale {
    float s, z, inv;
    bool live;                                                     // codes are not all 0
    uint32_t params;
    template <int kLanes> __device__ __forceinline__ void reduce(float lo, float hi, bool fine) {
        hi = fine ? hi : CUDART_INF_F;                             // carries the finding through the reduction
#pragma unroll
        for (int o = 1; o < kLanes; o <<= 1) {
            lo = fminf(lo, __shfl_xor_sync(0xFFFFFFFFu, lo, o));
            hi = fmaxf(hi, __shfl_xor_sync(0xFFFFFFFFu, hi, o));
        }
        z = bf16_down(lo);
        s = bf16_up_nonneg(__fdiv_rn(__fsub_rn(hi, z), 15.0f));
        const bool ok = hi <= 3.402823466e38f && z >= -3.402823466e38f && s <= 3.402823466e38f;
        s = s < 1.17549435e-38f ? 0.0f : s;
        live = ok && s > 0.0f;
        inv = __frcp_rn(s);
        params = ok ? (__float_as_uint(s) >> 16) | (__float_as_uint(z) & 0xFFFF0000u) : 0x7FFF7FFFu;
    }
    // a quad's codes: bits 0-7 channels 0 and 2, bits 16-23 channels 1 and 3
    static __device__ __forceinline__ uint32_t half_word(Two c, Two d) {
        return __float2uint_rz(fmaf(d.b, 1048576.0f, fmaf(c.b, 65536.0f, fmaf(d.a, 16.0f, c.a))));      // below 2^24: exact
    }
    __device__ __forceinline__ uint32_t word(const Two (&x)[4]) const {
        if (!live) return 0u;
        constexpr float kRound = 12582912.0f;                      // 1.5 * 2^23: adding it leaves the nearest whole number, ties to even
        Two c[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const Two d = add2(x[e], {-z, -z});
            Two q = mul2(d, {inv, inv});
            q = fma2(fma2(q, {-s, -s}, d), {inv, inv}, q);
            c[e] = add2(add2(q, {kRound, kRound}), {-kRound, -kRound});
        }
        if (!(s > 1e-27f && s < 1e30f)) {
#pragma unroll
            for (int e = 0; e < 4; ++e) c[e] = {rintf(__fdiv_rn(__fsub_rn(x[e].a, z), s)), rintf(__fdiv_rn(__fsub_rn(x[e].b, z), s))};
        }
        return half_word(c[0], c[1]) | half_word(c[2], c[3]) << 8;
    }
};
template <int kLanes> __device__ __forceinline__ void quantise_pair(const Two (&x)[4], const Two (&y)[4], uint32_t (&words)[2], uint32_t &params) {
    const Extrema ex(x), ey(y);
    Scale sc;
    sc.reduce<kLanes>(fminf(ex.lo, ey.lo), fmaxf(ex.hi, ey.hi), ex.fine && ey.fine);
    words[0] = sc.word(x);
    words[1] = sc.word(y);
    params = sc.params;
}

// The rotations that mix channels of other lanes or neighbouring ones: a lane holds eight channels in a row.
//
// kHeads heads of one kind (queries, keys or values) of one token per group of lanes.
template <typename DT, int D, bool kAppend, int kHeads>
__global__ void __launch_bounds__(kNormThreads, kHeads > 1 && sizeof(DT) == 2 && !kAppend ? 4 : 3) norm_rope_kernel(const NormArgs a) {
    constexpr int kLanes = D / 8;                                 // lanes of a row
    constexpr int kRunBytes = 16 * (D + 8);
    const int lane = threadIdx.x & (kLanes - 1);
    const uint32_t group = blockIdx.x * (kNormThreads / kLanes) + threadIdx.x / kLanes;
    const uint32_t t_raw = group / (uint32_t)a.chunks;
    const bool live = t_raw < (uint32_t)a.T;                      // whole groups: the shuffles below need every lane of the warp
    const int t = live ? (int)t_raw : a.T - 1;
    int chunk = (int)(group - t_raw * (uint32_t)a.chunks);
    // the chunks of a token: queries, keys, values
    const int kind = chunk < a.q_chunks ? 0 : !kAppend || chunk < a.q_chunks + a.k_chunks ? 1 : 2;
    chunk -= kind == 0 ? 0 : kind == 1 ? a.q_chunks : a.q_chunks + a.k_chunks;
    const int h0 = chunk * kHeads, heads = kind == 0 ? a.Hq : a.Hkv;
    const DT *src = static_cast<const DT *>(kind == 0 ? a.q : kind == 1 ? a.k : a.v);
    const long long st = kind == 0 ? a.q_t : kind == 1 ? a.k_t : a.v_t, sh = kind == 0 ? a.q_h : kind == 1 ? a.k_h : a.v_h;
    const bool vec = kind == 0 ? a.q_vec : kind == 1 ? a.k_vec : a.v_vec;
    const DT *weight = static_cast<const DT *>(kind == 0 ? a.q_weight : kind == 1 ? a.k_weight : nullptr);
    const bool rope = a.cos_sin != nullptr;                       // the same for the whole grid
    const int ch0 = lane * 8, ch1 = ch0 + 4;
    src += t * st;

    Quad<DT> raw[kHeads][2], wraw[2];
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
        const DT *row = src + min(h0 + i, heads - 1) * sh;
        raw[i][0].load(row + ch0, vec);
        raw[i][1].load(row + ch1, vec);
    }
    const int pos = a.positions ? a.positions[t] : 0;
    if (weight) {
        wraw[0].load(weight + ch0, a.w_vec);
        wraw[1].load(weight + ch1, a.w_vec);
    }
    const bool pad = pos < 0, beyond = rope && pos >= a.max_pos;
    const bool turned = rope && kind < 2 && ch0 < a.rot;
    Two c[4], s[4];                                               // angles: neighbouring pairs, the lane's four; else of all eight channels
    if (turned) {
        const int half = a.rot >> 1;
        const float *row = a.cos_sin + (long long)min(max(pos, 0), a.max_pos - 1) * a.rot;
        row += a.interleaved ? ch0 >> 1 : ch0 < half ? ch0 : ch0 - half;
        auto angles = [&](const float *p, Two &x, Two &y) {
            if (a.cs_vec) {
                const float4 v = __ldg(reinterpret_cast<const float4 *>(p));
                x = {v.x, v.y};
                y = {v.z, v.w};
            } else {
                x = {__ldg(p), __ldg(p + 1)};
                y = {__ldg(p + 2), __ldg(p + 3)};
            }
        };
        angles(row, c[0], c[1]);
        angles(row + half, s[0], s[1]);
        if (!a.interleaved) {
            angles(row + 4, c[2], c[3]);
            angles(row + half + 4, s[2], s[3]);
        }
    }
    // Sums of squares of the chunk's heads, then 1 / sqrt once for all of them: each of the first lanes takes one head's.
    // (Heads of all kinds may share a warp, and a warp's lanes go through the shuffles together.)
    float r[kHeads];
    if (__any_sync(0xFFFFFFFFu, weight != nullptr)) {
        float sum[kHeads];
#pragma unroll
        for (int i = 0; i < kHeads; ++i) {
            Two x[4];
            raw[i][0].get(x[0], x[1]);
            raw[i][1].get(x[2], x[3]);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = mul2(x[e], x[e]);
            sum[i] = __fadd_rn(__fadd_rn(__fadd_rn(x[0].a, x[0].b), __fadd_rn(x[1].a, x[1].b)),
                               __fadd_rn(__fadd_rn(x[2].a, x[2].b), __fadd_rn(x[3].a, x[3].b)));
        }
#pragma unroll
        for (int o = 1; o < kLanes; o <<= 1)
#pragma unroll
            for (int i = 0; i < kHeads; ++i) sum[i] = __fadd_rn(sum[i], __shfl_xor_sync(0xFFFFFFFFu, sum[i], o));
        float mine = 0.0f;
#pragma unroll
        for (int i = 0; i < kHeads; ++i) mine = i == 0 || (lane & (kHeads - 1)) == i ? sum[i] : mine;
        mine = __fdiv_rn(1.0f, __fsqrt_rn(__fadd_rn(__fmul_rn(mine, 1.0f / D), a.eps)));
#pragma unroll
        for (int i = 0; i < kHeads; ++i) r[i] = kHeads == 1 ? mine : __shfl_sync(0xFFFFFFFFu, mine, i, kLanes);
    }
    Two w[4];
    if (weight) {
        wraw[0].get(w[0], w[1]);
        wraw[1].get(w[2], w[3]);
    }
    const bool any_kept = kAppend && __any_sync(0xFFFFFFFFu, kind > 0);
    const long long slot = kAppend && kind > 0 ? a.slot[t] : -1;
    const bool kept = live && !pad && slot >= 0 && slot < a.n_slots;
    const long long block = kept ? block_of(slot, a.page) : 0;
    const int place = kept ? (int)(slot - block * a.page) : 0, tok = place & 15;
    // where this token lies in the cache: a head further is a page's worth of runs further
    const long long head_bytes = kAppend ? (long long)(a.page >> 4) * kRunBytes : 0;
    uint8_t *run0 = kAppend ? a.cache + (block * a.Hkv + h0) * head_bytes + (long long)(place >> 4) * kRunBytes : nullptr;
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
        const int h = h0 + i;
        Two x[4];
        raw[i][0].get(x[0], x[1]);
        raw[i][1].get(x[2], x[3]);
        if (weight) {
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = mul2(mul2(x[e], {r[i], r[i]}), w[e]);
        }
        if (rope) {
            if (a.interleaved) {
                if (turned) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float ce = e & 1 ? c[e >> 1].b : c[e >> 1].a, se = e & 1 ? s[e >> 1].b : s[e >> 1].a;
                        x[e] = add_products(mul2(x[e], {ce, ce}), mul2({x[e].b, x[e].a}, {-se, se}));
                    }
                }
            } else {
                const int hop = a.rot >> 4;                       // lanes between a channel and its partner
                const bool first = lane < hop;
                const int from = first ? lane + hop : lane < 2 * hop ? lane - hop : lane;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const Two o = {__shfl_sync(0xFFFFFFFFu, x[e].a, from, kLanes), __shfl_sync(0xFFFFFFFFu, x[e].b, from, kLanes)};
                    if (turned) {
                        x[e] = add_products(mul2(x[e], c[e]), mul2(o, first ? Two{-s[e].a, -s[e].b} : s[e]));      // a - b and a + (-b) are the same number
                    }
                }
            }
        }
        if (kind < 2 && (pad || beyond)) {
            const float v = pad ? 0.0f : CUDART_NAN_F;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = {v, v};
        }
        const bool mine = live && h < heads;
        if (kind == 0 || !kAppend) {
            DT *out = static_cast<DT *>(kind == 0 ? a.q_out : a.k_out);
            if (mine && out) {
                out += ((long long)t * heads + h) * D;
                Quad<DT>::store(out + ch0, x[0], x[1]);
                Quad<DT>::store(out + ch1, x[2], x[3]);
            }
        }
        if (kAppend && any_kept) {
            if constexpr (D <= 128) {
                if (kind == 1) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = Quad<DT>::rounded(x[e]);
                }
                const Extrema ex(x);
                Scale sc;
                sc.reduce<kLanes>(ex.lo, ex.hi, ex.fine);
                const uint32_t word = sc.word(x), params = sc.params;
                if (kept && h < heads) {
                    uint8_t *run = run0 + i * head_bytes;
                    *reinterpret_cast<uint32_t *>(run + (kind == 1 ? Kv4<D>::key_word(tok, lane) : Kv4<D>::kValueOff + Kv4<D>::value_word(tok, lane))) = word;
                    if (lane == 0) *reinterpret_cast<uint32_t *>(run + Kv4<D>::kParamOff + tok * 8 + (kind == 1 ? 0 : 4)) = params;
                }
            }
        }
    }
}

// The usual case: no rotation, or one of all channels or their first half with pairs half of that apart.  A lane holds the eight
// channels from ch0 and the eight that the rotation pairs with them (with rot = D / 2 the upper lanes hold the channels that are
// not turned in the same way), so a row takes D / 16 lanes, loads and stores are whole 16-byte vectors, nothing but the row's sum
// and extrema goes through shuffles, and each eight channels are a word of codes.  The lanes' sums meet in the order of a tree of
// neighbouring channels: up to `turning` lanes of either eight, then the two, then the rest.
template <typename DT, int D, bool kAppend, int kHeads>
__global__ void __launch_bounds__(kNormThreads, 3) norm_rope_paired_kernel(const NormArgs a) {
    constexpr int kLanes = D / 16;                                // lanes of a row
    constexpr int kRunBytes = 16 * (D + 8);
    const int lane = threadIdx.x & (kLanes - 1);
    const uint32_t group = blockIdx.x * (kNormThreads / kLanes) + threadIdx.x / kLanes;
    const uint32_t t_raw = group / (uint32_t)a.chunks;
    const bool live = t_raw < (uint32_t)a.T;                      // whole groups: the shuffles below need every lane of the warp
    const int t = live ? (int)t_raw : a.T - 1;
    int chunk = (int)(group - t_raw * (uint32_t)a.chunks);
    // the chunks of a token: queries, keys, values
    const int kind = chunk < a.q_chunks ? 0 : !kAppend || chunk < a.q_chunks + a.k_chunks ? 1 : 2;
    chunk -= kind == 0 ? 0 : kind == 1 ? a.q_chunks : a.q_chunks + a.k_chunks;
    const int h0 = chunk * kHeads, heads = kind == 0 ? a.Hq : a.Hkv;
    const DT *src = static_cast<const DT *>(kind == 0 ? a.q : kind == 1 ? a.k : a.v);
    const long long st = kind == 0 ? a.q_t : kind == 1 ? a.k_t : a.v_t, sh = kind == 0 ? a.q_h : kind == 1 ? a.k_h : a.v_h;
    const bool vec = kind == 0 ? a.q_vec : kind == 1 ? a.k_vec : a.v_vec;
    const DT *weight = static_cast<const DT *>(kind == 0 ? a.q_weight : kind == 1 ? a.k_weight : nullptr);
    const bool rope = a.cos_sin != nullptr;                       // the same for the whole grid
    const int turning = rope ? a.rot >> 4 : kLanes;               // lanes whose channels are turned
    const int ch0 = lane < turning ? lane * 8 : 8 * lane + 8 * turning, ch1 = ch0 + 8 * turning;

    Eight<DT> raw[kHeads][2], wraw[2];
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
        const DT *row = src + t * st + min(h0 + i, heads - 1) * sh;
        raw[i][0].load(row + ch0, vec);
        raw[i][1].load(row + ch1, vec);
    }
    const int pos = a.positions ? a.positions[t] : 0;
    if (weight) {
        wraw[0].load(weight + ch0, a.w_vec);
        wraw[1].load(weight + ch1, a.w_vec);
    }
    const bool pad = pos < 0, beyond = rope && pos >= a.max_pos;
    const bool turned = rope && kind < 2 && lane < turning;
    Two c[4], s[4];
    if (turned) {
        const float *row = a.cos_sin + (long long)min(max(pos, 0), a.max_pos - 1) * a.rot + ch0;
        Eight<float> cv, sv;
        cv.load(row, a.cs_vec);
        sv.load(row + (a.rot >> 1), a.cs_vec);
        cv.get(c);
        sv.get(s);
    }
    float r[kHeads];
    if (__any_sync(0xFFFFFFFFu, weight != nullptr)) {
        float sum0[kHeads], sum1[kHeads];
#pragma unroll
        for (int i = 0; i < kHeads; ++i) {
            Two x[4];
            raw[i][0].get(x);
            sum0[i] = square_sum(x);
            raw[i][1].get(x);
            sum1[i] = square_sum(x);
        }
#pragma unroll
        for (int o = 1; o < kLanes; o <<= 1) {
            if (o == turning) {
#pragma unroll
                for (int i = 0; i < kHeads; ++i) { sum0[i] = __fadd_rn(sum0[i], sum1[i]); sum1[i] = 0.0f; }
            }
#pragma unroll
            for (int i = 0; i < kHeads; ++i) {
                sum0[i] = __fadd_rn(sum0[i], __shfl_xor_sync(0xFFFFFFFFu, sum0[i], o));
                sum1[i] = __fadd_rn(sum1[i], __shfl_xor_sync(0xFFFFFFFFu, sum1[i], o));
            }
        }
        // 1 / sqrt once for all heads: each of the first lanes takes one head's
        float mine = 0.0f;
#pragma unroll
        for (int i = 0; i < kHeads; ++i) {
            sum0[i] = __fadd_rn(sum0[i], sum1[i]);                 // adds the zero where that has been done
            mine = i == 0 || (lane & (kHeads - 1)) == i ? sum0[i] : mine;
        }
        mine = __fdiv_rn(1.0f, __fsqrt_rn(__fadd_rn(__fmul_rn(mine, 1.0f / D), a.eps)));
#pragma unroll
        for (int i = 0; i < kHeads; ++i) r[i] = kHeads == 1 ? mine : __shfl_sync(0xFFFFFFFFu, mine, i, kLanes);
    }
    const bool any_kept = kAppend && __any_sync(0xFFFFFFFFu, kind > 0);
    const long long slot = kAppend && kind > 0 ? a.slot[t] : -1;
    const bool kept = live && !pad && slot >= 0 && slot < a.n_slots;
    const long long block = kept ? block_of(slot, a.page) : 0;
    const int place = kept ? (int)(slot - block * a.page) : 0, tok = place & 15;
    // where this token lies in the cache: a head further is a page's worth of runs further
    const long long head_bytes = kAppend ? (long long)(a.page >> 4) * kRunBytes : 0;
    uint8_t *run0 = kAppend ? a.cache + (block * a.Hkv + h0) * head_bytes + (long long)(place >> 4) * kRunBytes : nullptr;
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
        const int h = h0 + i;
        const bool mine = live && h < heads;
        Two x[4], y[4];
        raw[i][0].get(x);
        raw[i][1].get(y);
        if (weight) {
            Two w[4];
            wraw[0].get(w);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = mul2(mul2(x[e], {r[i], r[i]}), w[e]);
            wraw[1].get(w);
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = mul2(mul2(y[e], {r[i], r[i]}), w[e]);
        }
        if (turned) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {                          // a - b and a + (-b) are the same number
                const Two z = add_products(mul2(x[e], c[e]), mul2(y[e], {-s[e].a, -s[e].b}));
                y[e] = add_products(mul2(y[e], c[e]), mul2(x[e], s[e]));
                x[e] = z;
            }
        }
        if (kind < 2 && (pad || beyond)) {
            const float v = pad ? 0.0f : CUDART_NAN_F;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = y[e] = {v, v};
        }
        if (kind == 0 || !kAppend) {
            DT *out = static_cast<DT *>(kind == 0 ? a.q_out : a.k_out);
            if (mine && out) {
                out += ((long long)t * heads + h) * D;
                Eight<DT>::store(out + ch0, x);
                Eight<DT>::store(out + ch1, y);
            }
        }
        if (kAppend && any_kept) {
            if constexpr (D <= 128) {
                if (kind == 1) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x[e] = Quad<DT>::rounded(x[e]);
                        y[e] = Quad<DT>::rounded(y[e]);
                    }
                }
                uint32_t words[2], params;
                quantise_pair<kLanes>(x, y, words, params);
                if (kept && h < heads) {
                    uint8_t *run = run0 + i * head_bytes;
                    const int w0 = ch0 >> 3, w1 = ch1 >> 3;
                    *reinterpret_cast<uint32_t *>(run + (kind == 1 ? Kv4<D>::key_word(tok, w0) : Kv4<D>::kValueOff + Kv4<D>::value_word(tok, w0))) = words[0];
                    *reinterpret_cast<uint32_t *>(run + (kind == 1 ? Kv4<D>::key_word(tok, w1) : Kv4<D>::kValueOff + Kv4<D>::value_word(tok, w1))) = words[1];
                    if (lane == 0) *reinterpret_cast<uint32_t *>(run + Kv4<D>::kParamOff + tok * 8 + (kind == 1 ? 0 : 4)) = params;
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

// One word of key codes and one of value codes per lane: eight channels each.  8192 tokens of 8 heads of 128: 10 to 12 us for 42 MB read and
// written (6.5 at the copy's rate): a lane has one load of each in flight before it can store.
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
    DT *k_out = static_cast<DT *>(a.k_out) + row * D + lane * 8, *v_out = static_cast<DT *>(a.v_out) + row * D + lane * 8;
#pragma unroll
    for (int e = 0; e < 8; e += 4) {
        Quad<DT>::store(k_out + e, {k[e], k[e + 1]}, {k[e + 2], k[e + 3]});
        Quad<DT>::store(v_out + e, {v[e], v[e + 1]}, {v[e + 2], v[e + 3]});
    }
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
    // A long append is two launches: its queries alone need fewer registers and less code than keys and values, and so run
    // faster (8192 tokens of 40 + 2 x 8 heads of 128: 65 us instead of 74; 2048: 19.8 and 20.4; 1024: 12.5 and 12.2).
    if (kAppend && a.Hq > 0 && (long long)a.T * (a.Hq + 2 * a.Hkv) * (D / 16) > 148LL * 4096) {
        NormArgs q = a;
        q.Hkv = 0;
        const cudaError_t e = launch_norm_heads<DT, D, false>(q, st);
        if (e != cudaSuccess) return e;
        a.Hq = 0;
    }
    // Several heads to a group of lanes where there is more than a round or two of groups: a short call is the latency of one
    // group's chain, a long one wants loads in flight.  40 + 8 heads of 128, several and one: 64 tokens 2.5 and 2.3 us, 272: 3.5 and
    // 3.7, 512: 4.6 and 5.4, 8192: 47 and 71.  With the codes the chain is longer and registers are dearer (the forms of several heads keep 24
    // to 100 bytes a thread in memory): 512 tokens 8.1 and 7.2, 800: 9.8 and 10.5, 8192: 65 and 90.
    // Pairs save shuffles and read both halves of a row at once, which in long calls pays in bf16 only, and not where half of a head of
    // 128 is turned (8192 tokens, paired and not; bf16: 48 heads of 128 45 and 54 us, half turned 67 and 53; 40 of 64 19.1 and 21.1, half
    // turned 19.2 and 21.4; 20 of 256, half turned 40 and 46.  fp32: 40 of 64 35 and 33, half turned 65 and 33; 20 of 128 38 and 35).
    // Short calls are always better paired (64 tokens, bf16, 48 of 128: 2.6 and 3.3, half turned 3.0 and 3.2).
    const long long rows = (long long)a.T * (a.Hq + (kAppend ? 2 : 1) * a.Hkv), limit = 148LL * (kAppend ? 2048 : 512);
    const bool apart = sizeof(DT) == 4 || (D == 128 && a.cos_sin && a.rot == D / 2);
    const bool paired = (!apart || rows * (D / 16) <= limit) && (!a.cos_sin || (!a.interleaved && (a.rot == D || a.rot == D / 2)));
    const int lanes = paired ? D / 16 : D / 8;
    const bool wide = rows * lanes > limit;
    const int per = !wide ? 1 : paired ? 2 : 4;
    a.q_chunks = (a.Hq + per - 1) / per;
    a.k_chunks = (a.Hkv + per - 1) / per;
    a.chunks = a.q_chunks + (kAppend ? 2 : 1) * a.k_chunks;
    const long long groups = (long long)a.T * a.chunks, per_cta = kNormThreads / lanes;
    const unsigned grid = (unsigned)((groups + per_cta - 1) / per_cta);
    if (paired && wide) {
        if constexpr (sizeof(DT) == 2) norm_rope_paired_kernel<DT, D, kAppend, 2><<<grid, kNormThreads, 0, st>>>(a);
    } else if (paired)
        norm_rope_paired_kernel<DT, D, kAppend, 1><<<grid, kNormThreads, 0, st>>>(a);
    else if (wide)
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
