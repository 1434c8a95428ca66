// dsp_attn_kv4: attention of a step's tokens over the paged 4-bit cache.
#include <math.h>

#include "attn.cuh"
#include "attn_block.h"
#include "copy_ring.h"

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
// Pairs of fp32 numbers (two query rows) that go through the arithmetic together.
__device__ __forceinline__ void fma2(float &da, float &db, float s, float xa, float xb, float ya, float yb) {      // d = s x + y
    asm("{\n .reg .b64 s, x, y;\n mov.b64 s, {%2, %2};\n mov.b64 x, {%3, %4};\n mov.b64 y, {%5, %6};\n fma.rn.f32x2 y, s, x, y;\n mov.b64 {%0, %1}, y;\n}"
        : "=f"(da), "=f"(db) : "f"(s), "f"(xa), "f"(xb), "f"(ya), "f"(yb));
}
__device__ __forceinline__ void mul2(float &xa, float &xb, float s) {
    asm("{\n .reg .b64 s, x;\n mov.b64 s, {%2, %2};\n mov.b64 x, {%0, %1};\n mul.rn.f32x2 x, s, x;\n mov.b64 {%0, %1}, x;\n}" : "+f"(xa), "+f"(xb) : "f"(s));
}
__device__ __forceinline__ void add2(float &xa, float &xb, float ya, float yb) {
    asm("{\n .reg .b64 x, y;\n mov.b64 x, {%0, %1};\n mov.b64 y, {%2, %3};\n add.rn.f32x2 x, x, y;\n mov.b64 {%0, %1}, x;\n}" : "+f"(xa), "+f"(xb) : "f"(ya), "f"(yb));
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float y;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
    return y;
}

// Two codes as bf16 numbers 128 + code (0x4300 is 128, whose last mantissa bit is worth 1): (w >> 4i & 0x000F000F) | 0x43004300.
__device__ __forceinline__ uint32_t biased(uint32_t w, int i) {
    uint32_t y;
    asm("lop3.b32 %0, %1, 0x000F000F, 0x43004300, 0xEA;" : "=r"(y) : "r"(w >> (4 * i)));
    return y;
}
// A bulk copy into this CTA's shared memory, counted by a barrier there.
__device__ __forceinline__ void copy_bulk(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 :: "r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void expect_bytes(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" :: "r"(bar), "r"(bytes) : "memory");
}
// The same without their bias, and centred: code - 8, exactly.
__device__ __forceinline__ uint32_t centred(uint32_t x) {
    uint32_t y;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(x), "r"(0x43084308u));
    return y;
}
constexpr long long kWaitClocks = 4000000000LL;  // about two seconds: a wait that long has failed
__device__ __forceinline__ bool bytes_here(uint32_t bar, uint32_t parity) {
    long long t0 = 0;
    while (true) {
        uint32_t ok;
        asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
                     : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
        if (ok) return true;
        if (t0 == 0) t0 = clock64();
        else if (clock64() - t0 > kWaitClocks) return false;
    }
}
__device__ __forceinline__ uint4 lds128(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
    return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t at) {
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at));
    return v;
}

constexpr float kBias = 128.0f;

// A lane's codes of a run of 16 tokens, keys or values.
template <int D> struct Codes {
    uint4 v[D / 64];
    __device__ __forceinline__ void load(uint32_t at) {
#pragma unroll
        for (int i = 0; i < D / 64; ++i) v[i] = lds128(at + i * 512);
    }
    // word i of the keys of token r + 8 * hi
    __device__ __forceinline__ uint32_t key(int i, int hi) const {
        const uint4 &u = D == 128 ? v[D == 128 ? hi : 0] : v[0];
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

// The kernel for few query rows (a token, a short chain): the work that each byte of the cache needs is about as long as its way.
//
// Keys are the 16 rows of the matrix instruction and query rows its 8 columns: S^T = K Q^T, then
// O^T = V^T P^T with 16 value channels as rows, so 8 query rows fill an instruction, and the codes
// go from memory into the operand registers without a detour (the cache's order, dsp.h): four bits
// to bf16 is one masked OR (128 + code), with the bias and the scale left to the sums,
//     q . k = s (q . (128 + code)) + (z - 128 s) sum(q),
//     sum_u p v = sum_u (p s)(128 + code) - 136 sum_u (p s) + sum_u p (z + 8 s)
// where p s is rounded to bf16 as an operand and sum (p s) is formed from the rounded numbers by a
// matrix instruction with rows of ones (136 and the 8 s beside z centre the codes, which keeps the
// rounding error that of a centred value).  The bias leaves in every iteration: over a long stretch it
// would grow to thousands of times an output that averages over many tokens, and take its last bits.
//
// Each warp walks its own runs of 16 tokens with the next ones' copies in flight, and keeps its own
// running maximum: it moves only when a score passes it by 2^8 (the sums cannot overflow by that, and
// the division at the end takes it out), so most runs need no exchange between lanes for it.
// kW warps a CTA, kCtas CTAs an SM, kU runs an iteration, kStages iterations in the ring.
//
// Measured: one new token of 64 requests over up to 16384 tokens, 40 heads on 8 of 128: 179 us for 752 MB, 4.2 TB/s of the cache;
// the copies alone take 131.  A run's 2176 bytes need 273 instructions of a warp, which would be 84 us if one were issued every clock:
// the counters say one every second (51 %).  Sixteen warps an SM, as many as the registers hold, do not cover what an instruction waits
// for: per issue 1.6 warps wait for a result of the fixed kind, 1.1 for the ALU (60 % busy, the most of all units), 0.7 for memory.  64
// drafts of 32 tokens over 1023, 16 heads of 64: 64 us, bound by latency too (three CTAs an SM; a fourth spills: 72 us).  Some registers
// go to memory as it is: 8 rows of 128 44 bytes a thread, 16 rows 236, 32 rows 8 (of 64: 24).
//
// Before its first step a unit has kEnter places of the line for what every unit costs (queries, the first copies, the join of the
// warps): with none the CTAs that get many short units end last (64 requests of 32 new tokens over 1023, 16 heads of 64: 76 us
// instead of 65; where units are long they cost a little: one new token over 16384 177 us with none, 179 with them).
constexpr int kEnter = 4;
struct StreamRequest : Request {
    __device__ __forceinline__ int places() const { return steps + kEnter; }
    __device__ __forceinline__ long long length(int Hkv) const { return (long long)Hkv * tiles * places(); }
};

template <int D, int NT, int kW, int kCtas, int kU, int kStages>
__global__ void __launch_bounds__(kW * 32, kCtas) attn_stream_kernel(const AttnArgs a) {
    // how the values' bias leaves (see above): by a subtraction in the operand, once a code, or from the sums, once an output and
    // iteration; the latter is less work for few rows
    constexpr bool kCentred = NT >= 4;
    constexpr bool kQueriesShared = NT >= 4;                      // their fragments would not leave enough registers
    constexpr int kRows = 8 * NT, kStep = 16 * kU * kW, kKs = D / 16, kMt = D / 16;
    constexpr int kFrag = NT * kMt * 4 * 32;                      // floats of a partial output, in fragment order
    constexpr int kStage = kU * Kv4<D>::kRunBytes, kRing = kStages * kStage;
    // a ring of kStages iterations' codes for each warp; after a segment the same place takes its output
    extern __shared__ __align__(128) uint8_t s_dyn[];
    float (*s_o)[NT * kMt * 4][32] = reinterpret_cast<float (*)[NT * kMt * 4][32]>(s_dyn);
    __shared__ float s_m[kW][kRows], s_l[kW][kRows], s_top[kRows], s_sum[kRows];
    __shared__ __nv_bfloat16 *s_out[kRows];
    __shared__ uint64_t s_bars[kW][kStages];
    __shared__ int s_lim[kRows], s_query[kRows];                  // tokens that a row sees (before the bits), its query
    __shared__ long long s_scan[32];
    __shared__ LineStart s_line;
    __shared__ uint2 s_q[kQueriesShared ? NT : 1][kQueriesShared ? kKs : 1][32];
    __shared__ float s_qs[kRows];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = lane >> 2, c = lane & 3;
    grid_launch_dependents();                                     // the join's CTAs may come as soon as there is room
    if (threadIdx.x < kW * kStages)
        asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" :: "r"((uint32_t)__cvta_generic_to_shared(&s_bars[0][0] + threadIdx.x)) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    if (threadIdx.x == 0) a.split[blockIdx.x].last_cta = -1;
    enter_line<StreamRequest>(a, kRows, kStep, 1, s_scan, &s_line);
    long long at = s_line.begin;
    if (at >= s_line.end) return;
    const int runs_page = a.page >> 4;
    const long long head_bytes = (long long)runs_page * Kv4<D>::kRunBytes, block_bytes = head_bytes * a.Hkv;

    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(s_dyn) + warp * kRing;
    const uint32_t bars = (uint32_t)__cvta_generic_to_shared(&s_bars[warp][0]);
    CopyRing<kStages> order;
    bool lost = false;                                            // a copy has not come in time: the warp's rows get NaN, and nothing is fetched any more
    StreamRequest rq;
    long long before = s_line.before;
    rq.load(a, s_line.b, kRows, kStep);
    while (true) {
        const int unit = (int)((at - before) / rq.places()), off = (int)(at - before - (long long)unit * rq.places());
        const int h = unit / rq.tiles, tile = unit - h * rq.tiles;
        const int take = (int)min((long long)rq.places() - off, s_line.end - at);
        const int step0 = max(off - kEnter, 0), step1 = max(off + take - kEnter, 0);
        at += take;
        if (step0 == step1) break;                                // only places of the way in are left: the next CTA's unit
        const int row_first = tile * kRows, rows_here = min(rq.rows - row_first, kRows);
        // tokens below `safe` are seen by every row of the tile, none from `stop` on by any
        const int past = rq.kv - rq.n_new;                        // negative if more is new than there is
        const int i_first = row_first / a.group, i_last = (row_first + rows_here - 1) / a.group;
        if (threadIdx.x < kRows) {
            const int row = row_first + threadIdx.x, i = row / a.group;
            s_query[threadIdx.x] = i;
            s_lim[threadIdx.x] = row >= rq.rows ? 0 : a.mask_kind == DSP_MASK_CAUSAL ? min(rq.kv, past + i + 1) : rq.kv;
        }
        __syncthreads();
        const int safe = a.mask_kind == DSP_MASK_CAUSAL ? past + i_first + 1 : a.mask_kind == DSP_MASK_FULL ? rq.kv : past;
        const int stop = a.mask_kind == DSP_MASK_CAUSAL ? min(rq.kv, past + i_last + 1) : rq.kv;

        // this warp's runs: kU neighbouring ones an iteration, kW iterations' worth on from one to the next
        int run = (step0 * kW + warp) * kU;
        const int run_end = min(step1 * kW * kU, (max(stop, 0) + 15) >> 4);
        const int32_t *table = a.table + (long long)rq.b * a.table_stride;
        const uint8_t *head = a.cache + h * head_bytes;
        // Lane l looks up the run that is l / kU iterations ahead (its l % kU-th), the whole warp at once and a turn ahead; `valid`
        // and `joined` have a bit for each lane: its run's block exists, and the run after it lies next to it in the cache.
        const uint8_t *place = nullptr, *next_place = nullptr;
        int left = 0, next_run = run;
        uint32_t valid = 0u, joined = 0u;
        auto lookup = [&]() {
            place = next_place;
            valid = __ballot_sync(0xFFFFFFFFu, place != nullptr);
            const unsigned long long here = (unsigned long long)place;
            joined = __ballot_sync(0xFFFFFFFFu, here + Kv4<D>::kRunBytes == __shfl_down_sync(0xFFFFFFFFu, here, 1));
            left = 32;
            const int mine = next_run + (lane / kU) * (kW * kU) + lane % kU;
            next_place = nullptr;
            if (mine < run_end) {
                const int blk = runs_page == 1 ? mine : mine / runs_page, id = __ldg(table + blk);
                if (id >= 0 && id < a.n_blocks) next_place = head + id * block_bytes + (long long)(mine - blk * runs_page) * Kv4<D>::kRunBytes;
            }
            next_run += (32 / kU) * (kW * kU);
        };
        lookup();
        left = 0;
        uint32_t there = 0u;                                      // per stage and run: whether its block exists
        auto fetch = [&](int stage) {
            if (left == 0) lookup();
            const int from = 32 - left;
            constexpr uint32_t kAll = (1u << kU) - 1u;
            const uint32_t dst = ring + stage * kStage, bar = bars + 8 * stage, ok = (valid >> from) & kAll;
            there = (there & ~(kAll << (stage * kU))) | ok << (stage * kU);
            const uint8_t *src = (const uint8_t *)__shfl_sync(0xFFFFFFFFu, (unsigned long long)place, from);
            if (kU == 2 && ok == kAll && ((joined >> from) & 1u)) {      // neighbours: one piece
                if (lane == 0) {
                    expect_bytes(bar, kStage);
                    copy_bulk(dst, src, kStage, bar);
                }
            } else {
                const uint8_t *src2 = kU == 2 ? (const uint8_t *)__shfl_sync(0xFFFFFFFFu, (unsigned long long)place, from + kU - 1) : nullptr;
                if (lane == 0) {
                    expect_bytes(bar, __popc(ok) * Kv4<D>::kRunBytes);
                    if (ok & 1u) copy_bulk(dst, src, Kv4<D>::kRunBytes, bar);
                    if (kU == 2 && (ok & 2u)) copy_bulk(dst + Kv4<D>::kRunBytes, src2, Kv4<D>::kRunBytes, bar);
                }
            }
            left -= kU;
        };
        int ahead = run;                                          // the first copies are under way while the queries come
        order.restart();
#pragma unroll
        for (int i = 0; i < kStages - 1; ++i, ahead += kW * kU)
            if (ahead < run_end && !lost) fetch(i);
        auto load_queries = [&](int t, uint32_t (&x)[kKs * 2]) {
            const int row = row_first + t * 8 + r, i = row / a.group;
            const uint4 *src = reinterpret_cast<const uint4 *>(a.q + (long long)(rq.row0 + i) * a.q_t +
                                                               (long long)(h * a.group + row - i * a.group) * a.q_h + c * (D / 4));
#pragma unroll
            for (int k = 0; k < kKs / 2; ++k) {
                uint4 v = make_uint4(0u, 0u, 0u, 0u);
                if (row < rq.rows) v = __ldg(src + k);
                x[4 * k] = v.x; x[4 * k + 1] = v.y; x[4 * k + 2] = v.z; x[4 * k + 3] = v.w;
            }
        };
        auto query_sum = [&](const uint32_t (&x)[kKs * 2]) {
            float sum = 0.0f;
#pragma unroll
            for (int k = 0; k < kKs * 2; ++k) sum += bf16_lo(x[k]) + bf16_hi(x[k]);
            sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 1);
            return sum + __shfl_xor_sync(0xFFFFFFFFu, sum, 2);
        };
        // queries of lane's row r, its quarter of the channels in the cache's order
        uint32_t q[kQueriesShared ? 1 : NT][kKs * 2];
        float qs[NT][2];                                          // sums of the rows 2c, 2c + 1, times the scale
        if (kQueriesShared) {
            // as operand fragments, each by one warp
#pragma unroll
            for (int t = warp; t < NT; t += kW) {
                load_queries(t, q[0]);
#pragma unroll
                for (int j = 0; j < kKs; ++j) s_q[kQueriesShared ? t : 0][kQueriesShared ? j : 0][lane] = make_uint2(q[0][2 * j], q[0][2 * j + 1]);
                const float sum = query_sum(q[0]);
                if (c == 0) s_qs[t * 8 + r] = sum;
            }
            __syncthreads();
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 2; ++e) qs[t][e] = s_qs[t * 8 + 2 * c + e] * a.scale_log2;
        } else {
#pragma unroll
            for (int t = 0; t < NT; ++t) load_queries(t, q[kQueriesShared ? 0 : t]);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const float sum = query_sum(q[kQueriesShared ? 0 : t]);
#pragma unroll
                for (int e = 0; e < 2; ++e) qs[t][e] = __shfl_sync(0xFFFFFFFFu, sum, (2 * c + e) * 4) * a.scale_log2;
            }
        }
        // Scores are formed relative to the rows' reference -nb (base 2).  `unset`: rows of this lane (bit 2t + e) that have none
        // yet, because nothing of what they see has come; rows beyond the unit's keep 0.
        float o[NT][kMt][4], ps[kCentred ? 1 : NT][4] = {}, nb[NT][2], l[NT][2], zs[NT][2];
        uint32_t unset = 0u;
        bool started = false;                                     // nothing to rescale in the first iteration
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int j = 0; j < kMt; ++j) o[t][j][0] = o[t][j][1] = o[t][j][2] = o[t][j][3] = 0.0f;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                nb[t][e] = 0.0f; l[t][e] = 0.0f; zs[t][e] = 0.0f;
                unset |= (row_first + t * 8 + 2 * c + e < rq.rows ? 1u : 0u) << (2 * t + e);
            }
        }
        for (; run < run_end && !lost; run += kW * kU, ahead += kW * kU) {
            // the stage's bytes are here; where a wait runs out, what is still under way has to land before its place is used otherwise
            lost = !__all_sync(0xFFFFFFFFu, bytes_here(bars + 8 * order.stage, order.parity()));
            if (lost) {
#pragma unroll 1
                for (int left = order.under_way(run, ahead, run_end, kW * kU); left > 0; --left, order.used())
                    bytes_here(bars + 8 * order.stage, order.parity());
                break;
            }
            __syncwarp();                                         // all lanes have read the stage before
            if (ahead < run_end) fetch(order.before());
            const uint32_t codes = ring + order.stage * kStage + lane * 16, params = ring + order.stage * kStage + Kv4<D>::kParamOff + r * 8;
            const uint32_t here = there >> (order.stage * kU);
            order.used();
            // a run beyond the end or of no block leaves its operands at whatever the ring holds (codes are finite) and is not seen
            float s[kU][NT][4], va[kU][2], vz[kU][2];
#pragma unroll
            for (int x = 0; x < kU; ++x) {
                Codes<D> k;
                k.load(codes + x * Kv4<D>::kRunBytes);
#pragma unroll
                for (int t = 0; t < NT; ++t) s[x][t][0] = s[x][t][1] = s[x][t][2] = s[x][t][3] = 0.0f;
#pragma unroll
                for (int j = 0; j < kKs; ++j) {
                    const uint32_t w0 = k.key(j >> 1, 0), w1 = k.key(j >> 1, 1);
                    const int i = 2 * (j & 1);
                    const uint32_t a0 = biased(w0, i), a1 = biased(w1, i), a2 = biased(w0, i + 1), a3 = biased(w1, i + 1);
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        if (kQueriesShared) {
                            const uint2 b = s_q[kQueriesShared ? t : 0][kQueriesShared ? j : 0][lane];
                            mma_bf16(s[x][t], a0, a1, a2, a3, b.x, b.y);
                        } else {
                            mma_bf16(s[x][t], a0, a1, a2, a3, q[kQueriesShared ? 0 : t][2 * j], q[kQueriesShared ? 0 : t][2 * j + 1]);
                        }
                    }
                }
                // tokens r (e < 2) and r + 8: their scales, in base 2
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const uint2 p = lds64(params + x * Kv4<D>::kRunBytes + y * 64);
                    const float ks = bf16_lo(p.x), kz = bf16_hi(p.x);
                    const float ka = ks * a.scale_log2, kb = fmaf(-kBias, ks, kz);
                    va[x][y] = bf16_lo(p.y);
                    vz[x][y] = fmaf(8.0f, va[x][y], bf16_hi(p.y));
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        float c0, c1;
                        fma2(c0, c1, kb, qs[t][0], qs[t][1], nb[t][0], nb[t][1]);
                        fma2(s[x][t][2 * y], s[x][t][2 * y + 1], ka, s[x][t][2 * y], s[x][t][2 * y + 1], c0, c1);
                    }
                }
            }
            const bool whole = (run + kU) * 16 <= min(safe, run_end * 16) && (here & ((1u << kU) - 1)) == (1u << kU) - 1;
            uint32_t seen = 0xFFFFFFFFu;                          // bit (x NT + t) 4 + e
            if (!whole) {
                seen = 0u;
#pragma unroll
                for (int x = 0; x < kU; ++x)
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int u = (run + x) * 16 + r + 8 * (e >> 1), row = t * 8 + 2 * c + (e & 1);
                            bool ok = ((here >> x) & 1u) && run + x < run_end && u < s_lim[row];
                            if (a.mask_kind == DSP_MASK_BITS && ok && u >= past) {
                                const int j = u - past;
                                ok = j < a.words * 32 && ((__ldg(a.bits + (long long)(rq.row0 + s_query[row]) * a.words + (j >> 5)) >> (j & 31)) & 1u);
                            }
                            if (!ok) s[x][t][e] = -CUDART_INF_F;
                            seen |= (ok ? 1u : 0u) << ((x * NT + t) * 4 + e);
                        }
            }
            // A reference moves when a score passes it by 2^8, and is set by the first score that its row sees.
            float top = -CUDART_INF_F;
#pragma unroll
            for (int x = 0; x < kU; ++x)
#pragma unroll
                for (int t = 0; t < NT; ++t) top = max3(max3(top, s[x][t][0], s[x][t][1]), s[x][t][2], s[x][t][3]);
            if (__any_sync(0xFFFFFFFFu, top > 8.0f || unset != 0u)) {
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float row = fmaxf(s[0][t][e], s[0][t][e + 2]);
#pragma unroll
                        for (int x = 1; x < kU; ++x) row = max3(row, s[x][t][e], s[x][t][e + 2]);
                        row = fmaxf(row, __shfl_xor_sync(0xFFFFFFFFu, row, 4));
                        row = fmaxf(row, __shfl_xor_sync(0xFFFFFFFFu, row, 8));
                        row = fmaxf(row, __shfl_xor_sync(0xFFFFFFFFu, row, 16));
                        const bool first = (unset >> (2 * t + e)) & 1u;
                        const float by = (first ? row > -CUDART_INF_F : row > 8.0f) ? row : 0.0f;
                        const float keep = first ? 1.0f : ex2_approx(-by);      // a row without a reference has nothing to rescale
                        if (row > -CUDART_INF_F) unset &= ~(1u << (2 * t + e));
                        nb[t][e] -= by;
#pragma unroll
                        for (int x = 0; x < kU; ++x) { s[x][t][e] -= by; s[x][t][e + 2] -= by; }
                        if (started) {
                            l[t][e] *= keep;
                            zs[t][e] *= keep;
#pragma unroll
                            for (int j = 0; j < kMt; ++j) { o[t][j][e] *= keep; o[t][j][e + 2] *= keep; }
                        }
                    }
            }
            started = true;
#pragma unroll
            for (int x = 0; x < kU; ++x) {
                uint32_t p[NT][2];
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    float w[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[e] = ex2_approx(s[x][t][e]);
                    add2(l[t][0], l[t][1], w[0], w[1]);
                    add2(l[t][0], l[t][1], w[2], w[3]);
                    if (whole) {
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            fma2(zs[t][0], zs[t][1], vz[x][y], w[2 * y], w[2 * y + 1], zs[t][0], zs[t][1]);
                            mul2(w[2 * y], w[2 * y + 1], va[x][y]);
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const bool ok = (seen >> ((x * NT + t) * 4 + e)) & 1u;      // what is not seen is not multiplied: its scale may be NaN
                            zs[t][e & 1] += ok ? w[e] * vz[x][e >> 1] : 0.0f;
                            w[e] = ok ? w[e] * va[x][e >> 1] : 0.0f;
                        }
                    }
                    p[t][0] = transpose8x8(pack_bf16(w[0], w[1]));
                    p[t][1] = transpose8x8(pack_bf16(w[2], w[3]));
                    if (!kCentred) mma_bf16(ps[kCentred ? 0 : t], 0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u, p[t][0], p[t][1]);
                }
                Codes<D> v;
                v.load(codes + x * Kv4<D>::kRunBytes + Kv4<D>::kValueOff);
#pragma unroll
                for (int i = 0; i < kMt / 4; ++i) {
                    const uint32_t e0 = __byte_perm(v.val(i, 0, 0), v.val(i, 0, 1), 0x5410), o0 = __byte_perm(v.val(i, 0, 0), v.val(i, 0, 1), 0x7632);
                    const uint32_t e1 = __byte_perm(v.val(i, 1, 0), v.val(i, 1, 1), 0x5410), o1 = __byte_perm(v.val(i, 1, 0), v.val(i, 1, 1), 0x7632);
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        uint32_t a0 = biased(e0, y), a1 = biased(o0, y), a2 = biased(e1, y), a3 = biased(o1, y);
                        if (kCentred) { a0 = centred(a0); a1 = centred(a1); a2 = centred(a2); a3 = centred(a3); }
#pragma unroll
                        for (int t = 0; t < NT; ++t) mma_bf16(o[t][4 * i + y], a0, a1, a2, a3, p[t][0], p[t][1]);
                    }
                }
            }
            if (!kCentred) {
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    float (&sum)[4] = ps[kCentred ? 0 : t];
#pragma unroll
                    for (int j = 0; j < kMt; ++j) {
                        fma2(o[t][j][0], o[t][j][1], -(kBias + 8.0f), sum[0], sum[1], o[t][j][0], o[t][j][1]);
                        fma2(o[t][j][2], o[t][j][3], -(kBias + 8.0f), sum[0], sum[1], o[t][j][2], o[t][j][3]);
                    }
                    sum[0] = sum[1] = sum[2] = sum[3] = 0.0f;
                }
            }
        }
        __syncthreads();                                          // the rings' places become s_o
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
                if (lost) l[t][e] = CUDART_NAN_F;
                if (r == 0) {
                    s_m[warp][t * 8 + 2 * c + e] = (unset >> (2 * t + e)) & 1u ? -CUDART_INF_F : -nb[t][e];
                    s_l[warp][t * 8 + 2 * c + e] = l[t][e];
                }
            }
        __syncthreads();
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int row = t * 8 + 2 * c + e;
                float top = s_m[0][row];
#pragma unroll
                for (int w = 1; w < kW; ++w) top = fmaxf(top, s_m[w][row]);
                const float mine = s_m[warp][row], keep = mine == top ? 1.0f : ex2_approx(mine - top);
                const float off = zs[t][e];
#pragma unroll
                for (int j = 0; j < kMt; ++j) {
                    s_o[warp][(t * kMt + j) * 4 + e][lane] = (o[t][j][e] + off) * keep;
                    s_o[warp][(t * kMt + j) * 4 + e + 2][lane] = (o[t][j][e + 2] + off) * keep;
                }
                if (warp == t % kW && r == 0) {
                    float sum = 0.0f;
#pragma unroll
                    for (int w = 0; w < kW; ++w) sum += s_m[w][row] == top ? s_l[w][row] : s_l[w][row] * ex2_approx(s_m[w][row] - top);
                    const int rr = row_first + row, q_i = s_query[row];
                    s_top[row] = top;
                    s_sum[row] = sum;
                    s_out[row] = row < rows_here ? a.out + ((long long)(rq.row0 + q_i) * a.Hq + h * a.group + rr - q_i * a.group) * D : nullptr;
                }
            }
        __syncthreads();
        const bool starts = step0 == 0, ends = step1 == rq.steps;
        float *part = a.part + ((long long)blockIdx.x * 2 + (starts ? 1 : 0)) * (kFrag + 2 * kRows);
        // a thread takes kJ neighbouring channel pairs of a row
        constexpr int kAll = NT * kMt * 64 / (kW * 32), kJ = kAll >= 4 ? 4 : kAll >= 2 ? 2 : 1;
#pragma unroll
        for (int i = threadIdx.x; i < NT * kMt * 64 / kJ; i += kW * 32) {
            const int ln = i & 31, e = (i >> 5) & 1, tj = (i >> 6) * kJ, t = tj / kMt, j = tj % kMt;
            const int row = t * 8 + 2 * (ln & 3) + e;
            float x[kJ] = {}, y[kJ] = {};
#pragma unroll
            for (int w = 0; w < kW; ++w)
#pragma unroll
                for (int z = 0; z < kJ; ++z) {
                    x[z] += s_o[w][(tj + z) * 4 + e][ln];
                    y[z] += s_o[w][(tj + z) * 4 + e + 2][ln];
                }
            if (starts && ends) {
                __nv_bfloat16 *out = s_out[row];
                if (out) {
                    const float sum = s_sum[row], inv = sum == 0.0f ? 0.0f : __fdividef(1.0f, sum);
                    uint32_t v[kJ];
#pragma unroll
                    for (int z = 0; z < kJ; ++z) v[z] = sum == 0.0f ? 0u : pack_bf16(x[z] * inv, y[z] * inv);
                    out += (ln >> 2) * (D / 8) + 8 * (j >> 2) + 2 * (j & 3);
                    if constexpr (kJ == 4) *reinterpret_cast<uint4 *>(out) = make_uint4(v[0], v[1], v[2], v[3]);
                    else if constexpr (kJ == 2) *reinterpret_cast<uint2 *>(out) = make_uint2(v[0], v[1]);
                    else *reinterpret_cast<uint32_t *>(out) = v[0];
                }
            } else {
#pragma unroll
                for (int z = 0; z < kJ; ++z) {
                    part[((tj + z) * 4 + e) * 32 + ln] = x[z];
                    part[((tj + z) * 4 + e + 2) * 32 + ln] = y[z];
                }
                if (j == 0 && (ln >> 2) == 0) {
                    part[kFrag + row] = s_top[row];
                    part[kFrag + kRows + row] = s_sum[row];
                }
            }
        }
        if (starts && !ends && threadIdx.x == 0) {
            SplitUnit u;
            u.b = rq.b; u.h = h; u.tile = tile;
            u.last_cta = cta_of(before + (long long)(h * rq.tiles + tile + 1) * rq.places() - 1, s_line.total, s_line.ctas);
            a.split[blockIdx.x] = u;
        }
        if (at >= s_line.end) break;
        while (at >= before + rq.length(a.Hkv)) {
            before += rq.length(a.Hkv);
            rq.load(a, rq.b + 1, kRows, kStep);
        }
        // the places of s_o, written and read as ordinary memory, are the copies' again
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncthreads();
    }
}

// Joins the partial results of one unit that crossed the shares of several CTAs, in their order.  A long request alone may
// leave one from every CTA: they are taken 16 or 32 at a time, all loads of a turn in flight together.  (Ordinary loads: the parts are
// written while this kernel's CTAs already wait, and a read-only load is for what nobody writes as long as its kernel runs.)
constexpr int kJoinThreads = 256;
template <int D, int NT>
__global__ void __launch_bounds__(kJoinThreads) attn_join_kernel(const AttnArgs a) {
    constexpr int kRows = 8 * NT, kMt = D / 16, kFrag = NT * kMt * 4 * 32, kPart = kFrag + 2 * kRows, kJoinTurn = NT == 1 ? 32 : 16;
    constexpr int kPairs = NT * kMt * 2 * 32 / kJoinThreads > 0 ? NT * kMt * 2 * 32 / kJoinThreads : 1;
    __shared__ float s_f[kJoinTurn][kRows], s_keep[kRows], s_m[kRows], s_l[kRows];
    grid_dependency_wait();
    const SplitUnit u = a.split[blockIdx.x];
    if (u.last_cta < 0) return;
    const int first = blockIdx.x, n = u.last_cta - first + 1, tid = threadIdx.x;
    const int row0 = max(a.cu[u.b], 0), n_new = max(min(min(a.cu[u.b + 1], a.T) - row0, a.max_new), 0);
    // part i: the unit's first CTA left its second place, the others their first
    const float *base = a.part + (long long)first * 2 * kPart;
    if (tid < kRows) {
        s_m[tid] = -CUDART_INF_F;
        s_l[tid] = 0.0f;
    }
    float x[kPairs] = {}, y[kPairs] = {};
    for (int i0 = 0; i0 < n; i0 += kJoinTurn) {
        __syncthreads();
        for (int i = tid; i < kJoinTurn * kRows; i += kJoinThreads) {
            const int w = i / kRows;
            s_f[w][i % kRows] = i0 + w < n ? base[(long long)((i0 + w) * 2 + (i0 + w == 0 ? 1 : 0)) * kPart + kFrag + i % kRows] : -CUDART_INF_F;
        }
        __syncthreads();
        if (tid < kRows) {
            const float before = s_m[tid];
            float top = before, l[kJoinTurn];
#pragma unroll
            for (int w = 0; w < kJoinTurn; ++w) {
                top = fmaxf(top, s_f[w][tid]);
                l[w] = i0 + w < n ? base[(long long)((i0 + w) * 2 + (i0 + w == 0 ? 1 : 0)) * kPart + kFrag + kRows + tid] : 0.0f;
            }
            const float keep = before == top ? 1.0f : ex2_approx(before - top);
            float sum = s_l[tid] * keep;
#pragma unroll
            for (int w = 0; w < kJoinTurn; ++w) {
                const float m = s_f[w][tid], f = i0 + w >= n ? 0.0f : m == top ? 1.0f : ex2_approx(m - top);
                s_f[w][tid] = f;
                sum = fmaf(l[w], f, sum);
            }
            s_keep[tid] = keep;
            s_m[tid] = top;
            s_l[tid] = sum;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kPairs; ++k) {
            const int i = tid + k * kJoinThreads, ln = i & 31, q = i >> 5, e = q & 1, tj = q >> 1;
            if (tj >= NT * kMt) break;
            const int row = (tj / kMt) * 8 + 2 * (ln & 3) + e, at = (tj * 4 + e) * 32 + ln;
            float vx[kJoinTurn], vy[kJoinTurn];
#pragma unroll
            for (int w = 0; w < kJoinTurn; ++w) {
                const float *p = base + (long long)((i0 + w) * 2 + (i0 + w == 0 ? 1 : 0)) * kPart + at;
                vx[w] = i0 + w < n ? p[0] : 0.0f;
                vy[w] = i0 + w < n ? p[64] : 0.0f;
            }
            x[k] *= s_keep[row];
            y[k] *= s_keep[row];
#pragma unroll
            for (int w = 0; w < kJoinTurn; ++w) {
                x[k] = fmaf(vx[w], s_f[w][row], x[k]);
                y[k] = fmaf(vy[w], s_f[w][row], y[k]);
            }
        }
    }
#pragma unroll
    for (int k = 0; k < kPairs; ++k) {
        const int i = tid + k * kJoinThreads, ln = i & 31, q = i >> 5, e = q & 1, tj = q >> 1, j = tj % kMt;
        if (tj >= NT * kMt) break;
        const int row = (tj / kMt) * 8 + 2 * (ln & 3) + e, rr = u.tile * kRows + row;
        if (rr >= n_new * a.group) continue;
        const float sum = s_l[row], inv = 1.0f / sum;
        const int q_i = rr / a.group, ch = (ln >> 2) * (D / 8) + 8 * (j >> 2) + 2 * (j & 3);
        *reinterpret_cast<uint32_t *>(a.out + ((long long)(row0 + q_i) * a.Hq + u.h * a.group + rr - q_i * a.group) * D + ch) =
            sum == 0.0f ? 0u : pack_bf16(x[k] * inv, y[k] * inv);
    }
}

// Launch shape of a call, from what the host knows of it.
struct Shape {
    bool block;                                  // the kernel for many rows
    int nt, warps, ctas_sm, unroll, grid;
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
    // Query rows are columns of the matrix instruction in the kernel for few rows, which unpacks codes in every warp, and a tile of 128 in
    // the other.  32 rows over 8192 tokens, 16 requests, 8 key heads of 128: 71 us for few rows, 97 for many (of 64: 48 and 75).  Beyond 32
    // the sums no longer fit the registers, and the codes are unpacked once for every 32 rows: 64 rows 122 and 104 (of 64: 85 and 92).
    s.block = rows > 32;
    if (s.block) {
        s.nt = s.warps = s.unroll = 0;
        s.ctas_sm = 1;
        s.grid = sm_count();
        s.part_bytes = attn_block_part_bytes(D);
        return s;
    }
    // 64 requests over 8192, 8 key heads of 128: 8 rows 104 us in one column group, 131 in two; 16 rows 127 us in two, 214 in four
    s.nt = rows <= 8 ? 1 : rows <= 16 ? 2 : 4;
    s.warps = 4;
    s.ctas_sm = s.nt == 1 ? 4 : s.nt == 2 || D == 64 ? 3 : 2;
    s.unroll = s.nt == 4 ? 1 : 2;
    s.grid = sm_count() * s.ctas_sm;
    s.part_bytes = ((size_t)s.nt * D * 8 + 16 * s.nt) * sizeof(float);
    return s;
}

template <int D, int NT, int kW, int kCtas, int kU, int kStages>
cudaError_t launch_stream(const AttnArgs &a, int grid, cudaStream_t st) {
    constexpr int ring = kW * kStages * kU * Kv4<D>::kRunBytes, outs = kW * NT * (D / 16) * 4 * 32 * 4, smem = ring > outs ? ring : outs;
    static std::atomic<unsigned long long> done{0};
    cudaError_t e = allow_shared(attn_stream_kernel<D, NT, kW, kCtas, kU, kStages>, smem, done);
    if (e != cudaSuccess) return e;
    attn_stream_kernel<D, NT, kW, kCtas, kU, kStages><<<grid, kW * 32, smem, st>>>(a);
    e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    return launch_dependent(attn_join_kernel<D, NT>, (unsigned)grid, kJoinThreads, 0, st, a, true);
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
    if (!isfinite(scale * kLog2e)) return DSP_ERR_INVALID_ARG;
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
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (s.block) {
        DSP_CUDA_TRY(attn_block_launch(a, D, s.grid, st));
        return DSP_OK;
    }
    // no more CTAs than the line can have steps, as far as the host knows the lengths
    const long long tokens = (long long)max_blocks * page_size, rows = (long long)a.max_new * a.group;
    const long long most = (long long)B * Hkv * ((rows + 8 * s.nt - 1) / (8 * s.nt)) * ((tokens + 16 * s.unroll * s.warps - 1) / (16 * s.unroll * s.warps));
    const int grid = (int)(most < s.grid ? most : s.grid);
    cudaError_t e;
    if (D == 64)
        e = s.nt == 1 ? launch_stream<64, 1, 4, 4, 2, 3>(a, grid, st) : s.nt == 2 ? launch_stream<64, 2, 4, 3, 2, 3>(a, grid, st)
                      : launch_stream<64, 4, 4, 3, 1, 4>(a, grid, st);
    else
        e = s.nt == 1 ? launch_stream<128, 1, 4, 4, 2, 3>(a, grid, st) : s.nt == 2 ? launch_stream<128, 2, 4, 3, 2, 3>(a, grid, st)
                      : launch_stream<128, 4, 4, 2, 1, 4>(a, grid, st);
    DSP_CUDA_TRY(e);
    return DSP_OK;
}
