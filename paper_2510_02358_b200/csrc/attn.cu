// dsp_attn_kv4: attention of a step's tokens over the paged 4-bit cache.
#include <math.h>

#include "attn.cuh"

namespace dsp {
namespace {

__device__ __forceinline__ void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&p);
}
// Two codes as bf16 numbers 128 + code (0x4300 is 128, whose last mantissa bit is worth 1).
__device__ __forceinline__ uint32_t biased(uint32_t w, int i) { return code_pair(w, i) | 0x43004300u; }

constexpr float kBias = 128.0f;

// A run of 16 tokens of one key head on its way through a warp's registers.
template <int D> struct Run {
    static constexpr int kVec = D / 64;          // 16-byte vectors of codes a lane holds, for keys and for values
    uint4 k[kVec], v[kVec];
    uint2 p[2];                                  // scales and offsets of the tokens r and r + 8
    bool there;                                  // false: no such block, nothing was read
    __device__ __forceinline__ void load(const uint8_t *run, int lane, bool ok) {
        there = ok;
        if (ok) {
#pragma unroll
            for (int i = 0; i < kVec; ++i) k[i] = ldg_stream(run + i * 512 + lane * 16);
#pragma unroll
            for (int i = 0; i < kVec; ++i) v[i] = ldg_stream(run + Kv4<D>::kValueOff + i * 512 + lane * 16);
            p[0] = __ldg(reinterpret_cast<const uint2 *>(run + Kv4<D>::kParamOff) + (lane >> 2));
            p[1] = __ldg(reinterpret_cast<const uint2 *>(run + Kv4<D>::kParamOff) + (lane >> 2) + 8);
        } else {
#pragma unroll
            for (int i = 0; i < kVec; ++i) k[i] = v[i] = make_uint4(0u, 0u, 0u, 0u);
            p[0] = p[1] = make_uint2(0u, 0u);
        }
    }
    // word i of the keys of token r + 8 * hi
    __device__ __forceinline__ uint32_t key(int i, int hi) const {
        const uint4 &u = D == 128 ? k[D == 128 ? hi : 0] : k[0];
        const int at = D == 128 ? i : 2 * hi + i;
        return at == 0 ? u.x : at == 1 ? u.y : at == 2 ? u.z : u.w;
    }
    // word i of the values of the tokens 2c + 8 * hi and 2c + 1 + 8 * hi
    __device__ __forceinline__ uint32_t val(int i, int hi, int odd) const {
        const uint4 &u = D == 128 ? v[D == 128 ? hi : 0] : v[0];
        const int at = D == 128 ? 2 * odd + i : 2 * hi + odd;
        return at == 0 ? u.x : at == 1 ? u.y : at == 2 ? u.z : u.w;
    }
};

// The kernel for few query rows (a token, a short chain): bound by the bytes of the cache.
//
// Keys are the 16 rows of the matrix instruction and query rows its 8 columns: S^T = K Q^T, then
// O^T = V^T P^T with 16 value channels as rows, so 8 query rows fill an instruction, and the codes
// go from memory into the operand registers without a detour (the cache's order, dsp.h): four bits
// to bf16 is one masked OR (128 + code), with the bias and the scale left to the sums,
//     q . k = s (q . (128 + code)) + (z - 128 s) sum(q),
//     sum_u p v = sum_u (p s)(128 + code) - 136 sum_u (p s) + sum_u p (z + 8 s)
// where p s is rounded to bf16 as an operand and sum (p s) is formed from the rounded numbers by a
// matrix instruction with rows of ones (so the bias leaves exactly; 136 and the 8 s beside z centre
// the codes, which keeps the rounding error that of a centred value).
//
// Each warp walks its own runs of 16 tokens with the next run's loads in flight, and keeps its own
// running maximum: it moves only when a score passes it by 2^8 (the sums cannot overflow by that, and
// the division at the end takes it out), so most runs need no exchange between lanes for it.
template <int D, int NT, int kW, int kCtas>
__global__ void __launch_bounds__(kW * 32, kCtas) attn_stream_kernel(const AttnArgs a) {
    constexpr int kRows = 8 * NT, kStep = 16 * kW, kKs = D / 16, kMt = D / 16;
    constexpr int kFrag = NT * kMt * 4 * 32;                      // floats of a partial output, in fragment order
    __shared__ float s_o[kW][NT * kMt * 4][32];
    __shared__ float s_m[kW][kRows], s_l[kW][kRows];
    __shared__ long long s_scan[32];
    __shared__ LineStart s_line;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = lane >> 2, c = lane & 3;
    if (threadIdx.x == 0) a.split[blockIdx.x].last_cta = -1;
    enter_line(a, kRows, kStep, s_scan, &s_line);
    long long at = s_line.begin;
    const long long end = s_line.end, total = s_line.total;
    if (at >= end) return;
    const int runs_page = a.page >> 4;
    const long long head_bytes = (long long)runs_page * Kv4<D>::kRunBytes, block_bytes = head_bytes * a.Hkv;

    Request rq;
    long long before = s_line.before;
    rq.load(a, s_line.b, kRows, kStep);
    while (true) {
        const int unit = (int)((at - before) / rq.steps), step0 = (int)(at - before - (long long)unit * rq.steps);
        const int h = unit / rq.tiles, tile = unit - h * rq.tiles;
        const int step1 = (int)min((long long)rq.steps, step0 + (end - at));
        const int row_first = tile * kRows, rows_here = min(rq.rows - row_first, kRows);
        // queries of lane's row r, its quarter of the channels in the cache's order
        uint32_t q[NT][kKs * 2];
        float qs[NT][2];
        int lim[NT][2];                                           // tokens that rows 2c, 2c+1 see (before the bits)
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int row = row_first + t * 8 + r;
            float sum = 0.0f;
            if (row < rq.rows) {
                const int i = row / a.group;
                const uint4 *src = reinterpret_cast<const uint4 *>(a.q + (long long)(rq.row0 + i) * a.q_t +
                                                                   (long long)(h * a.group + row - i * a.group) * a.q_h + c * (D / 4));
#pragma unroll
                for (int k = 0; k < kKs / 2; ++k) {
                    const uint4 x = __ldg(src + k);
                    q[t][4 * k] = x.x; q[t][4 * k + 1] = x.y; q[t][4 * k + 2] = x.z; q[t][4 * k + 3] = x.w;
                }
            } else {
#pragma unroll
                for (int k = 0; k < kKs * 2; ++k) q[t][k] = 0u;
            }
#pragma unroll
            for (int k = 0; k < kKs * 2; ++k) sum += bf16_lo(q[t][k]) + bf16_hi(q[t][k]);
            sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 1);
            sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 2);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                qs[t][e] = __shfl_sync(0xFFFFFFFFu, sum, (2 * c + e) * 4);
                const int row_e = row_first + t * 8 + 2 * c + e;
                lim[t][e] = row_e >= rq.rows ? 0
                            : a.mask_kind == DSP_MASK_CAUSAL ? min(rq.kv, rq.kv - rq.n_new + row_e / a.group + 1) : rq.kv;
            }
        }
        // tokens below `safe` are seen by every row of the tile, none from `stop` on by any
        const int past = rq.kv - rq.n_new;                        // negative if more is new than there is
        const int i_first = row_first / a.group, i_last = (row_first + rows_here - 1) / a.group;
        const int safe = a.mask_kind == DSP_MASK_CAUSAL ? past + i_first + 1 : a.mask_kind == DSP_MASK_FULL ? rq.kv : past;
        const int stop = a.mask_kind == DSP_MASK_CAUSAL ? min(rq.kv, past + i_last + 1) : rq.kv;

        float o[NT][kMt][4], ps[NT][4], m[NT][2], nm[NT][2], l[NT][2], zs[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int j = 0; j < kMt; ++j) o[t][j][0] = o[t][j][1] = o[t][j][2] = o[t][j][3] = 0.0f;
            ps[t][0] = ps[t][1] = ps[t][2] = ps[t][3] = 0.0f;
#pragma unroll
            for (int e = 0; e < 2; ++e) { m[t][e] = -CUDART_INF_F; nm[t][e] = 0.0f; l[t][e] = 0.0f; zs[t][e] = 0.0f; }
        }
        // this warp's runs: run0, run0 + kW, ...; their blocks are looked up two runs ahead, loaded one ahead
        int run = step0 * kW + warp;
        const int run_end = min(step1 * kW, (max(stop, 0) + 15) >> 4);
        const int hop_blk = kW / runs_page, hop_sub = kW - hop_blk * runs_page;
        int blk = run / runs_page, sub = run - blk * runs_page;
        const int32_t *table = a.table + (long long)rq.b * a.table_stride;
        const uint8_t *head = a.cache + h * head_bytes;
        auto advance = [&]() {
            blk += hop_blk;
            sub += hop_sub;
            if (sub >= runs_page) { sub -= runs_page; ++blk; }
        };
        Run<D> next;
        int id = -1, id_sub = 0;
        if (run < run_end) {
            const int first_id = table[blk];
            next.load(head + first_id * block_bytes + (long long)sub * Kv4<D>::kRunBytes, lane, first_id >= 0 && first_id < a.n_blocks);
            advance();
            if (run + kW < run_end) { id = table[blk]; id_sub = sub; }
        }
        for (; run < run_end; run += kW) {
            const Run<D> cur = next;
            if (run + kW < run_end) {
                next.load(head + id * block_bytes + (long long)id_sub * Kv4<D>::kRunBytes, lane, id >= 0 && id < a.n_blocks);
                advance();
                if (run + 2 * kW < run_end) { id = table[blk]; id_sub = sub; }
            }
            float s[NT][4];
#pragma unroll
            for (int t = 0; t < NT; ++t) s[t][0] = s[t][1] = s[t][2] = s[t][3] = 0.0f;
#pragma unroll
            for (int j = 0; j < kKs; ++j) {
                const uint32_t w0 = cur.key(j >> 1, 0), w1 = cur.key(j >> 1, 1);
                const int i = 2 * (j & 1);
                const uint32_t a0 = biased(w0, i), a1 = biased(w1, i), a2 = biased(w0, i + 1), a3 = biased(w1, i + 1);
#pragma unroll
                for (int t = 0; t < NT; ++t) mma_bf16(s[t], a0, a1, a2, a3, q[t][2 * j], q[t][2 * j + 1]);
            }
            // tokens r (e < 2) and r + 8: their scales, in base 2
            float ka[2], kb[2], va[2], vz[2];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const float ks = bf16_lo(cur.p[x].x), kz = bf16_hi(cur.p[x].x);
                ka[x] = ks * a.scale_log2;
                kb[x] = fmaf(-kBias, ks, kz) * a.scale_log2;
                va[x] = bf16_lo(cur.p[x].y);
                vz[x] = fmaf(8.0f, va[x], bf16_hi(cur.p[x].y));
            }
            const bool whole = run * 16 + 16 <= safe && cur.there;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[t][e] = fmaf(ka[e >> 1], s[t][e], kb[e >> 1] * qs[t][e & 1]);
            uint32_t seen = 0xFFFFFFFFu;                          // bit 4t + e
            if (!whole) {
                seen = 0u;
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int u = run * 16 + r + 8 * (e >> 1);
                        bool ok = cur.there && u < lim[t][e & 1];
                        if (a.mask_kind == DSP_MASK_BITS && ok && u >= past) {
                            const int j = u - past, i = (row_first + t * 8 + 2 * c + (e & 1)) / a.group;
                            ok = j < a.words * 32 && ((__ldg(a.bits + (long long)(rq.row0 + i) * a.words + (j >> 5)) >> (j & 31)) & 1u);
                        }
                        if (!ok) s[t][e] = -CUDART_INF_F;
                        seen |= (ok ? 1u : 0u) << (4 * t + e);
                    }
            }
            bool move = false;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) move = move || s[t][e] > m[t][e & 1] + 8.0f;
            if (__any_sync(0xFFFFFFFFu, move)) {
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float top = fmaxf(s[t][e], s[t][e + 2]);
                        top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 4));
                        top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 8));
                        top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 16));
                        top = fmaxf(top, m[t][e]);
                        const float keep = m[t][e] == top ? 1.0f : ex2_approx(m[t][e] - top);
                        m[t][e] = top;
                        nm[t][e] = top == -CUDART_INF_F ? 0.0f : -top;
                        l[t][e] *= keep;
                        zs[t][e] *= keep;
                        ps[t][e] *= keep;
#pragma unroll
                        for (int j = 0; j < kMt; ++j) { o[t][j][e] *= keep; o[t][j][e + 2] *= keep; }
                    }
            }
            uint32_t p[NT][2];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                float w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    w[e] = ex2_approx(s[t][e] + nm[t][e & 1]);
                    l[t][e & 1] += w[e];
                }
                if (whole) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        zs[t][e & 1] = fmaf(w[e], vz[e >> 1], zs[t][e & 1]);
                        w[e] *= va[e >> 1];
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const bool ok = (seen >> (4 * t + e)) & 1u;      // what is not seen is not multiplied: its scale may be NaN
                        zs[t][e & 1] += ok ? w[e] * vz[e >> 1] : 0.0f;
                        w[e] = ok ? w[e] * va[e >> 1] : 0.0f;
                    }
                }
                p[t][0] = transpose8x8(pack_bf16(w[0], w[1]));
                p[t][1] = transpose8x8(pack_bf16(w[2], w[3]));
                mma_bf16(ps[t], 0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u, p[t][0], p[t][1]);
            }
#pragma unroll
            for (int i = 0; i < kMt / 4; ++i) {
                const uint32_t e0 = __byte_perm(cur.val(i, 0, 0), cur.val(i, 0, 1), 0x5410), o0 = __byte_perm(cur.val(i, 0, 0), cur.val(i, 0, 1), 0x7632);
                const uint32_t e1 = __byte_perm(cur.val(i, 1, 0), cur.val(i, 1, 1), 0x5410), o1 = __byte_perm(cur.val(i, 1, 0), cur.val(i, 1, 1), 0x7632);
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const uint32_t a0 = biased(e0, x), a1 = biased(o0, x), a2 = biased(e1, x), a3 = biased(o1, x);
#pragma unroll
                    for (int t = 0; t < NT; ++t) mma_bf16(o[t][4 * i + x], a0, a1, a2, a3, p[t][0], p[t][1]);
                }
            }
        }
        // the warps' results: common maximum, then one sum per output in the order of the warps
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) {
                    l[t][e] += __shfl_xor_sync(0xFFFFFFFFu, l[t][e], x);
                    zs[t][e] += __shfl_xor_sync(0xFFFFFFFFu, zs[t][e], x);
                }
                if (r == 0) {
                    s_m[warp][t * 8 + 2 * c + e] = m[t][e];
                    s_l[warp][t * 8 + 2 * c + e] = l[t][e];
                }
            }
        __syncthreads();
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float top = s_m[0][t * 8 + 2 * c + e];
#pragma unroll
                for (int w = 1; w < kW; ++w) top = fmaxf(top, s_m[w][t * 8 + 2 * c + e]);
                const float keep = m[t][e] == top ? 1.0f : ex2_approx(m[t][e] - top);
                const float off = zs[t][e] - (kBias + 8.0f) * ps[t][e];
#pragma unroll
                for (int j = 0; j < kMt; ++j) {
                    s_o[warp][(t * kMt + j) * 4 + e][lane] = (o[t][j][e] + off) * keep;
                    s_o[warp][(t * kMt + j) * 4 + e + 2][lane] = (o[t][j][e + 2] + off) * keep;
                }
            }
        __syncthreads();
        const bool starts = step0 == 0, ends = step1 == rq.steps;
        float *part = a.part + ((long long)blockIdx.x * 2 + (starts ? 1 : 0)) * (kFrag + 2 * kRows);
        for (int i = threadIdx.x; i < NT * kMt * 2 * 32; i += kW * 32) {
            const int ln = i & 31, k = i >> 5, e = k & 1, tj = k >> 1, t = tj / kMt, j = tj - t * kMt;
            const int row = t * 8 + 2 * (ln & 3) + e;
            float x = 0.0f, y = 0.0f, sum = 0.0f, top = s_m[0][row];
#pragma unroll
            for (int w = 1; w < kW; ++w) top = fmaxf(top, s_m[w][row]);
#pragma unroll
            for (int w = 0; w < kW; ++w) {
                x += s_o[w][tj * 4 + e][ln];
                y += s_o[w][tj * 4 + e + 2][ln];
                sum += s_m[w][row] == top ? s_l[w][row] : s_l[w][row] * ex2_approx(s_m[w][row] - top);
            }
            if (starts && ends) {
                if (row < rows_here) {
                    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
                    const int rr = row_first + row, q_i = rr / a.group;
                    const int ch = (ln >> 2) * (D / 8) + 8 * (j >> 2) + 2 * (j & 3);
                    *reinterpret_cast<uint32_t *>(a.out + ((long long)(rq.row0 + q_i) * a.Hq + h * a.group + rr - q_i * a.group) * D + ch) =
                        sum == 0.0f ? 0u : pack_bf16(x * inv, y * inv);
                }
            } else {
                part[(tj * 4 + e) * 32 + ln] = x;
                part[(tj * 4 + e + 2) * 32 + ln] = y;
                if (j == 0 && (ln >> 2) == 0) {
                    part[kFrag + row] = top;
                    part[kFrag + kRows + row] = sum;
                }
            }
        }
        at += step1 - step0;
        if (starts && !ends && threadIdx.x == 0) {
            SplitUnit u;
            u.b = rq.b; u.h = h; u.tile = tile;
            u.last_cta = cta_of(at - step1 + rq.steps - 1, total, s_line.ctas);
            a.split[blockIdx.x] = u;
        }
        if (at >= end) break;
        while (at >= before + rq.length(a.Hkv)) {
            before += rq.length(a.Hkv);
            rq.load(a, rq.b + 1, kRows, kStep);
        }
        __syncthreads();                                          // s_o and s_m are written anew
    }
}

// Joins the partial results of one unit that crossed the shares of several CTAs, in their order.
template <int D, int NT>
__global__ void __launch_bounds__(128) attn_join_kernel(const AttnArgs a) {
    constexpr int kRows = 8 * NT, kMt = D / 16, kFrag = NT * kMt * 4 * 32;
    grid_dependency_wait();
    const SplitUnit u = a.split[blockIdx.x];
    if (u.last_cta < 0) return;
    const int first = blockIdx.x, n = u.last_cta - first + 1;
    const int row0 = max(a.cu[u.b], 0), n_new = max(min(min(a.cu[u.b + 1], a.T) - row0, a.max_new), 0);
    auto part_of = [&](int i) { return a.part + ((long long)(first + i) * 2 + (i == 0 ? 1 : 0)) * (kFrag + 2 * kRows); };
    for (int i = threadIdx.x; i < NT * kMt * 2 * 32; i += 128) {
        const int ln = i & 31, k = i >> 5, e = k & 1, tj = k >> 1, t = tj / kMt, j = tj - t * kMt;
        const int row = t * 8 + 2 * (ln & 3) + e, rr = u.tile * kRows + row;
        if (rr >= n_new * a.group) continue;
        float top = -CUDART_INF_F, x = 0.0f, y = 0.0f, sum = 0.0f;
        for (int w = 0; w < n; ++w) top = fmaxf(top, part_of(w)[kFrag + row]);
        for (int w = 0; w < n; ++w) {
            const float *p = part_of(w);
            const float m = p[kFrag + row], f = m == top ? 1.0f : ex2_approx(m - top);
            x = fmaf(p[(tj * 4 + e) * 32 + ln], f, x);
            y = fmaf(p[(tj * 4 + e + 2) * 32 + ln], f, y);
            sum = fmaf(p[kFrag + kRows + row], f, sum);
        }
        const float inv = 1.0f / sum;
        const int q_i = rr / a.group, ch = (ln >> 2) * (D / 8) + 8 * (j >> 2) + 2 * (j & 3);
        *reinterpret_cast<uint32_t *>(a.out + ((long long)(row0 + q_i) * a.Hq + u.h * a.group + rr - q_i * a.group) * D + ch) =
            sum == 0.0f ? 0u : pack_bf16(x * inv, y * inv);
    }
}

// Launch shape of a call, from what the host knows of it.
struct Shape {
    int nt, warps, ctas_sm, grid;
    size_t part_bytes;
};

int sm_count() {
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) n = 148;
    return n;
}

Shape shape_of(int32_t D, int32_t Hq, int32_t Hkv, int32_t max_new) {
    Shape s;
    const long long rows = (long long)max_new * (Hq / Hkv);
    s.nt = rows <= 8 ? 1 : 2;
    s.warps = s.nt == 1 ? 8 : 4;
    s.ctas_sm = s.nt == 1 ? 2 : 3;
    s.grid = sm_count() * s.ctas_sm;
    s.part_bytes = ((size_t)s.nt * D * 8 + 16 * s.nt) * sizeof(float);
    return s;
}

template <int D, int NT, int kW, int kCtas>
cudaError_t launch_stream(const AttnArgs &a, int grid, cudaStream_t st) {
    attn_stream_kernel<D, NT, kW, kCtas><<<grid, kW * 32, 0, st>>>(a);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    return launch_dependent(attn_join_kernel<D, NT>, (unsigned)grid, 128, 0, st, a, true);
}

}  // namespace
}  // namespace dsp

extern "C" int32_t dsp_attn_kv4_workspace_bytes(int32_t B, int32_t T, int32_t Hq, int32_t Hkv, int32_t D, int32_t max_new,
                                                size_t *bytes) {
    using namespace dsp;
    if (!bytes || B < 0 || T < 0 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0 || max_new < 1) return DSP_ERR_INVALID_ARG;
    if ((D != 64 && D != 128) || B > 65535 || T > (1 << 24) || Hq > 4096) return DSP_ERR_UNSUPPORTED;
    const Shape s = shape_of(D, Hq, Hkv, max_new);
    *bytes = align_up(s.grid * sizeof(SplitUnit), 256) + align_up(2 * s.grid * s.part_bytes, 256);
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
    const Shape s = shape_of(D, Hq, Hkv, max_new);
    AttnArgs a = {};
    a.q = static_cast<const __nv_bfloat16 *>(q);
    a.q_t = q_stride_t; a.q_h = q_stride_h;
    a.B = B; a.T = T; a.Hq = Hq; a.Hkv = Hkv; a.group = Hq / Hkv;
    a.cache = static_cast<const uint8_t *>(cache); a.n_blocks = n_blocks; a.page = page_size;
    a.table = block_table; a.table_stride = table_stride; a.max_blocks = max_blocks;
    a.kv_len = kv_len; a.cu = cu_new;
    a.max_new = max_new < T ? max_new : T;
    a.scale_log2 = scale * kLog2e;
    a.mask_kind = mask_kind; a.bits = mask_bits; a.words = mask_words;
    a.out = static_cast<__nv_bfloat16 *>(out);
    a.split = static_cast<SplitUnit *>(workspace);
    a.part = reinterpret_cast<float *>(static_cast<char *>(workspace) + align_up(s.grid * sizeof(SplitUnit), 256));
    // no more CTAs than the line can have steps, as far as the host knows the lengths
    const long long tokens = (long long)max_blocks * page_size, rows = (long long)a.max_new * a.group;
    const long long most = (long long)B * Hkv * ((rows + 8 * s.nt - 1) / (8 * s.nt)) * ((tokens + 16 * s.warps - 1) / (16 * s.warps));
    const int grid = (int)(most < s.grid ? most : s.grid);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (D == 64)
        e = s.nt == 1 ? launch_stream<64, 1, 8, 2>(a, grid, st) : launch_stream<64, 2, 4, 3>(a, grid, st);
    else
        e = s.nt == 1 ? launch_stream<128, 1, 8, 2>(a, grid, st) : launch_stream<128, 2, 4, 3>(a, grid, st);
    DSP_CUDA_TRY(e);
    return DSP_OK;
}
