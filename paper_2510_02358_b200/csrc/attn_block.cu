// The kernel of dsp_attn_kv4 for many query rows (verified blocks and trees times the heads of a group,
// prompts): bound by the tensor cores.
//
// One CTA per SM.  A unit is up to 256 query rows of one key head against a stretch of the cache; its
// rows are two tiles of 128 that share every key and value tile, or, with at most 128 rows, one tile
// whose even and odd token tiles go to the two halves of the CTA.  Either way there are two slots, each
// with a 128 x D output in tensor memory and two buffers of 128 x 64 scores (512 columns together): the
// tensor cores form the scores of a slot's next half tile while its last one is exponentiated, so the
// softmax warps, which are the slowest part, need not wait for them.
//
//   warps 0-7   softmax, four per slot, one thread per query row: maximum, exponentials, weights in fp16
//               back into the scores' columns as the second product's operand
//   warps 8-15  the tiles' codes (a run of 16 tokens each, keys then values): 16-byte loads one tile
//               ahead in registers, four bits to fp16 values, swizzled stores; two stages of each
//   warps 16-17 one lane each issues the products of a slot: S = Q K^T, O += P V
//
// Here a cached number is expanded once for 128 or 256 rows, so it becomes a whole value on the way
// (code * scale + offset, one rounding): folding the scales into the sums, as the kernel for few rows
// does, would cost each score more than that.  The operands are fp16, whose 11 bits leave the result's
// own rounding to bf16 as the error that counts (0.0017 of an output in the mean; with bf16 operands
// it was 0.0035).  What fp16's range does not hold is brought into it by powers of two: a row of queries
// by its largest number, taken back with the softmax scale; a key whose largest number lies outside
// 2^-4 .. 2^15 by that, its scores being multiplied back (k_mul).  Values are multiplied by 64, and the 16
// tokens of a run that holds one outside 2^-10 .. 2^9 go through bf16 operands instead (wide_runs), with the
// 64 in their weights.
//
// The running maximum moves only when a row's scores pass it by 2^8, and only then is the output in
// tensor memory rescaled (by the softmax warps, between two products of their slot).
//
// Measured: a chunk of 2 x 2048 new tokens over 8200, 40 heads on 8 of 128: 719 us among other calls, 780 TFLOP/s, and 656 us, 855
// TFLOP/s, where it alone is repeated (a plain matrix product: 1670); trees of 65 over 8192, 16 requests: 151 us.  A wide token tile takes
// about 5000 clocks, of which the tensor cores need 2560 (a product of 64 scores columns 48, bound by shared memory, one with the weights
// 64), the softmax warps 3900 and the fill warps 3400; of a form that took 674 us a copy without exponentials took as long, one without
// unpacking 626.  The loop from weights over the output's product and the next scores to the next weights is what bounds it: scores and
// weights of a half tile share their columns, and tensor memory has no others.  (96 registers a thread; 12 bytes of them go to memory.)
//
// Tokens that nobody may see (beyond the length, of a missing block) become zeros, and those whose scale
// or offset is NaN too, with a bit beside the tile: the rows that see such a token get a NaN score.
#include <cuda_fp16.h>

#include "attn.cuh"
#include "attn_block.h"

namespace dsp {
namespace {

constexpr int kSoftWarps = 8, kFillWarps = 8, kProductWarps = 2;
constexpr int kBlockThreads = (kSoftWarps + kFillWarps + kProductWarps) * 32;
constexpr int kTile = 128;                       // query rows of a slot, tokens of a tile
constexpr int kHalf = kTile / 2;                 // tokens whose scores are formed and exponentiated at once
constexpr int kRunsTile = kTile / 16;
constexpr long long kWaitClocks = 4000000000LL;  // about two seconds: a wait that long has failed
// Weights are formed as 2^(score - maximum + 7): at most 2^15, since a score passes the maximum by no more than 2^8, and whole fp16
// numbers down to 2^-21 of it.  Beside one dominant token the others' weights are small, and without the 7 they lost their last bits
// (at 2^-25 of it 1.3% of the output).  Sums and outputs carry the same 2^7, so it leaves with the division.
constexpr float kWeightUp = 7.0f;

// ---------------------------------------------------------------- tensor cores and barriers (PTX)
__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint32_t bar, int count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(bar) : "memory"); }
__device__ __forceinline__ bool bar_test(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0u;
}
// False when the wait has run out here or in another warp of the CTA.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int *dead) {
    if (bar_test(bar, parity)) return true;
    const long long t0 = clock64();
    while (!bar_test(bar, parity)) {
        if (*dead || clock64() - t0 > kWaitClocks) {
            *dead = 1;
            return false;
        }
    }
    return true;
}
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int *dead) {
    return __all_sync(0xFFFFFFFFu, bar_wait(bar, parity, dead));
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// Products and commits are issued by the lane whose `lead` is set; the rest of the warp passes by.  The lane is picked by a
// predicate and not by a branch: in a branch that only some lanes take, every operand has to be moved to the uniform registers
// that these instructions want, one at a time (measured: 120 clocks per product instead of 40).
__device__ __forceinline__ uint32_t elected() {
    uint32_t ok;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xFFFFFFFF;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(ok));
    return ok;
}
__device__ __forceinline__ void commit_to(uint32_t bar, uint32_t lead) {
    asm volatile("{\n .reg .pred e;\n setp.ne.u32 e, %1, 0;\n"
                 " @e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}" :: "r"(bar), "r"(lead) : "memory");
}
// Operand tiles lie in shared memory as blocks of 64 channels: [block][row][128 bytes], the 16-byte
// pieces of a row exchanged by its number modulo 8 (the 128-byte swizzle).  The same bytes serve as an
// operand contracted over the channels (queries, keys) and as one contracted over the rows (values).
__device__ __forceinline__ uint64_t tile_desc(uint32_t addr, uint32_t lead_bytes, uint32_t stride_bytes) {
    return (uint64_t)((addr & 0x3FFFF) >> 4) | (uint64_t)(lead_bytes >> 4) << 16 | (uint64_t)(stride_bytes >> 4) << 32 |
           (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
constexpr uint32_t kProduct = 1u << 4 | (uint32_t)(kTile >> 4) << 24;      // fp32 sums, fp16 operands, 128 rows
constexpr uint32_t kWithBf16 = 1u << 7 | 1u << 10;                         // bf16 operands instead
__device__ __forceinline__ void product_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add, uint32_t lead) {
    asm volatile("{\n .reg .pred p, e;\n setp.ne.u32 p, %4, 0;\n setp.ne.u32 e, %5, 0;\n"
                 " @e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
                 :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add), "r"(lead) : "memory");
}
__device__ __forceinline__ void product_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add, uint32_t lead) {
    asm volatile("{\n .reg .pred p, e;\n setp.ne.u32 p, %4, 0;\n setp.ne.u32 e, %5, 0;\n"
                 " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
                 :: "r"(d), "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)add), "r"(lead) : "memory");
}
__device__ __forceinline__ void tmem_load32(uint32_t at, float (&x)[32]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7]),
                   "=f"(x[8]), "=f"(x[9]), "=f"(x[10]), "=f"(x[11]), "=f"(x[12]), "=f"(x[13]), "=f"(x[14]), "=f"(x[15]),
                   "=f"(x[16]), "=f"(x[17]), "=f"(x[18]), "=f"(x[19]), "=f"(x[20]), "=f"(x[21]), "=f"(x[22]), "=f"(x[23]),
                   "=f"(x[24]), "=f"(x[25]), "=f"(x[26]), "=f"(x[27]), "=f"(x[28]), "=f"(x[29]), "=f"(x[30]), "=f"(x[31])
                 : "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_store4(uint32_t at, const uint32_t (&x)[4]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1,%2,%3,%4};" :: "r"(at), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]) : "memory");
}
// The registers pass through the wait, so that nothing uses them before it.
__device__ __forceinline__ void tmem_loaded(float (&x)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(x[0]), "+f"(x[1]), "+f"(x[2]), "+f"(x[3]), "+f"(x[4]), "+f"(x[5]), "+f"(x[6]), "+f"(x[7]),
                   "+f"(x[8]), "+f"(x[9]), "+f"(x[10]), "+f"(x[11]), "+f"(x[12]), "+f"(x[13]), "+f"(x[14]), "+f"(x[15]),
                   "+f"(x[16]), "+f"(x[17]), "+f"(x[18]), "+f"(x[19]), "+f"(x[20]), "+f"(x[21]), "+f"(x[22]), "+f"(x[23]),
                   "+f"(x[24]), "+f"(x[25]), "+f"(x[26]), "+f"(x[27]), "+f"(x[28]), "+f"(x[29]) , "+f"(x[30]), "+f"(x[31]) :: "memory");
}
// Eight columns, waited for.
__device__ __forceinline__ void tmem_load8(uint32_t at, float (&x)[8]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];\n tcgen05.wait::ld.sync.aligned;"
                 : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7]) : "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_store8(uint32_t at, const float (&x)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 :: "r"(at), "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]) : "memory");
}
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void pair_barrier(int id, int threads) { asm volatile("bar.sync %0, %1;" :: "r"(id), "r"(threads) : "memory"); }

// ------------------------------------------------------------------------------- cut of the work
// A request's units: tiles of 256 rows, for each tile its key heads.  A token tile of a unit with more
// than 128 rows counts kWide on the line, of one with fewer kNarrow: it has half the products but the
// same keys and values to expand (measured: about 4000 clocks against 5000).  Before its first token a unit has kEnter places of the line
// for what every unit costs, its queries and its output: with none the shares of many short units took longer than others (16
// requests of 65 new tokens over 8192, 40 heads on 8: 167 us instead of 150; the chunk of 2 x 2048 over 8200: 658 and 657).
constexpr int kWide = 4, kNarrow = 3, kEnter = 12;
struct BlockRequest {
    int b, n_new, kv, rows, row0, group, tiles;
    bool causal;
    __device__ __forceinline__ void load(const AttnArgs &a, int b_, int, int) {
        Request r;
        r.load(a, b_, 2 * kTile, kTile);
        b = b_; n_new = r.n_new; kv = r.kv; rows = r.rows; row0 = r.row0; tiles = r.tiles;
        group = a.group;
        causal = a.mask_kind == DSP_MASK_CAUSAL;
    }
    __device__ __forceinline__ int rows_of(int tile) const { return min(rows - tile * 2 * kTile, 2 * kTile); }
    __device__ __forceinline__ int weight(int tile) const { return rows_of(tile) > kTile ? kWide : kNarrow; }
    __device__ __forceinline__ int steps(int tile) const {
        const int last = (tile * 2 * kTile + rows_of(tile) - 1) / group;
        const int end = causal ? min(kv, kv - n_new + last + 1) : kv;
        return max(1, (end + kTile - 1) / kTile);
    }
    __device__ __forceinline__ int places(int tile) const { return steps(tile) * weight(tile) + kEnter; }
    __device__ __forceinline__ long long length(int Hkv) const {
        if (!causal) {
            const long long whole = rows / (2 * kTile), rest = rows - whole * 2 * kTile, n = max(1, (kv + kTile - 1) / kTile);
            return Hkv * (n * (kWide * whole + (rest > kTile ? kWide : rest > 0 ? kNarrow : 0)) + (long long)kEnter * tiles);
        }
        long long n = 0;
        for (int t = 0; t < tiles; ++t) n += places(t);
        return n * Hkv;
    }
};

// One CTA's way along its share of the line: a segment is the steps step0 .. step1-1 of a unit.
struct Walk {
    BlockRequest rq;
    long long at, end, total;
    int ctas;
    int tile, h, off;                            // unit, and how far the share's place is into it
    int step0, step1, steps, weight;
    __device__ __forceinline__ void enter(const AttnArgs &a, const LineStart &s) {
        at = s.begin; end = s.end; total = s.total; ctas = s.ctas;
        tile = h = off = 0;
        if (at >= end) return;
        rq.load(a, s.b, 0, 0);
        long long rest = at - s.before;
        while (true) {
            const long long len = (long long)rq.places(tile) * a.Hkv;
            if (rest < len) break;
            rest -= len;
            ++tile;
        }
        const int unit = rq.places(tile);
        h = (int)(rest / unit);
        off = (int)(rest - (long long)h * unit);
    }
    // The next segment; false at the share's end.
    __device__ __forceinline__ bool next(const AttnArgs &a) {
        while (at < end) {
            steps = rq.steps(tile);
            weight = rq.weight(tile);
            const int len = steps * weight + kEnter, take = (int)min((long long)(len - off), end - at);
            step0 = max(off - kEnter, 0) / weight;
            step1 = max(off + take - kEnter, 0) / weight;
            at += take;
            off += take;
            if (step1 > step0) return true;
            leave(a);
        }
        return false;
    }
    // On to the next unit (after a segment has been used).
    __device__ __forceinline__ void leave(const AttnArgs &a) {
        if (at >= end) return;
        off = 0;
        if (++h < a.Hkv) return;
        h = 0;
        if (++tile < rq.tiles) return;
        tile = 0;
        do {
            rq.load(a, rq.b + 1, 0, 0);
        } while (rq.tiles == 0);
    }
    __device__ __forceinline__ bool wide() const { return weight == kWide; }
    __device__ __forceinline__ int row_first() const { return tile * 2 * kTile; }
};
// Every warp has a walk of its own in shared memory (its state is not worth registers); lane 0 takes the steps.
__device__ __forceinline__ void walk_enter(Walk &w, const AttnArgs &a, const LineStart &s, int lane) {
    if (lane == 0) w.enter(a, s);
    __syncwarp();
}
__device__ __forceinline__ bool walk_next(Walk &w, const AttnArgs &a, int lane) {
    __syncwarp();
    bool more = false;
    if (lane == 0) more = w.next(a);
    __syncwarp();
    return __shfl_sync(0xFFFFFFFFu, more, 0);
}
__device__ __forceinline__ void walk_leave(Walk &w, const AttnArgs &a, int lane) {
    __syncwarp();
    if (lane == 0) w.leave(a);
}

struct Bars {
    uint64_t key_full[2], key_empty[2], val_full[2], val_empty[2];
    uint64_t score_full[4], weight_ready[4];     // [slot * 2 + buffer]
    uint64_t out_free[2];                        // [slot] its last product with the weights has ended
    uint64_t query_ready, out_done;
    uint64_t ended;                              // every product that was issued
};
struct __align__(16) Info {                      // beside a token tile, one bit per token
    uint32_t there[4], poison[4], scaled[4];     // 16 bits from each fill warp: there is such a token, it holds NaN, its k_mul is not 1
    float k_mul[kTile];
    uint8_t wide_runs[8];                        // whether a run's values are bf16
    uint8_t odd[8];                              // whether anything of the above is other than usual in a run
};

// ------------------------------------------------------------------------------- codes to values
// Scale and offset of a token, both in both halves; fp16 numbers take a second scale for the codes that come 16 times as large.
struct Affine {
    uint32_t s, s16, z;
};
__device__ __forceinline__ uint32_t twice_f16(float x) {
    const __half2 h = __float2half2_rn(x);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ uint32_t twice_bf16(float x) {
    const __nv_bfloat162 h = __float2bfloat162_rn(x);
    return *reinterpret_cast<const uint32_t *>(&h);
}
// Eight channels.  fp16: 0x6400 is 1024 and its last bit is worth 1, so a masked OR makes 1024 + code or 1024 + 16 code; taking
// 1024 off is exact, and code * s + z is rounded once.
__device__ __forceinline__ uint4 values_f16(uint32_t w, const Affine &a) {
    uint32_t v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t c;
        if (i & 1) asm("lop3.b32 %0, %1, 0x00F000F0, 0x64006400, 0xEA;" : "=r"(c) : "r"(w));
        else asm("lop3.b32 %0, %1, 0x000F000F, 0x64006400, 0xEA;" : "=r"(c) : "r"(w));
        asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(c) : "r"(c), "r"(0x64006400u));
        asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(v[i]) : "r"(c), "r"(i & 1 ? a.s16 : a.s), "r"(a.z));
        if (i == 1) w >>= 8;
    }
    return make_uint4(v[0], v[1], v[2], v[3]);
}
// bf16: the same with 128 + code.
__device__ __forceinline__ uint4 values_bf16(uint32_t w, const Affine &a) {
    uint32_t v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t c;
        asm("lop3.b32 %0, %1, 0x000F000F, 0x43004300, 0xEA;" : "=r"(c) : "r"(w >> (4 * i)));
        asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(c) : "r"(c), "r"(0x43004300u));
        asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(v[i]) : "r"(c), "r"(a.s), "r"(a.z));
    }
    return make_uint4(v[0], v[1], v[2], v[3]);
}
// Four pairs of bf16 numbers without infinities: the sum of a scale and an offset near the range's end may pass it, and rows that do
// not see the token multiply it by 0.
__device__ __forceinline__ uint4 finite_bf16(uint4 v) {
    uint32_t *p = &v.x;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        asm("min.bf16x2 %0, %0, %1;\n max.bf16x2 %0, %0, %2;" : "+r"(p[i]) : "r"(0x7F7F7F7Fu), "r"(0xFF7FFF7Fu));
    return v;
}
__device__ __forceinline__ void store16(uint32_t at, const uint4 &v) {
    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" :: "r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ uint4 load16(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
// The largest number that a head of scale and offset p (bf16 each) may hold, in magnitude.
__device__ __forceinline__ float largest(uint32_t p) { return fmaxf(fabsf(bf16_hi(p)), fabsf(fmaf(15.0f, bf16_lo(p), bf16_hi(p)))); }
// Values are multiplied by it on the way in (those of bf16 runs, which may lie near the range's end, through their weights), outputs by
// its inverse on the way out.
constexpr float kValueMul = 64.0f;
__device__ __forceinline__ bool value_fits(uint32_t p) {
    const float top = largest(p);
    return top == 0.0f || (top >= 0.0009765625f && top < 512.0f);
}
__device__ __forceinline__ bool not_finite(uint32_t p) { return (p & 0x7FFFu) >= 0x7F80u || (p & 0x7FFF0000u) >= 0x7F800000u; }
// Where the 16-byte piece `piece` (channels 8 piece ..) of row t lies in an operand tile.
__device__ __forceinline__ uint32_t piece_at(int t, int piece) {
    return (uint32_t)((piece >> 3) * (kTile * 128) + t * 128 + (((piece & 7) ^ (t & 7)) << 4));
}

// A fill warp's run of a tile: 16 tokens, keys and values.
template <int D> struct Fill {
    static constexpr int kVec = D / 64;
    uint4 k[kVec], v[kVec];
    uint2 kp[2];                                 // scales and offsets of the tokens r and r + 8
    uint4 vp[2];                                 // of the tokens 2c, 2c+1 and 2c+8, 2c+9
    bool ok_k, ok_v;
    __device__ __forceinline__ void load_keys(const uint8_t *run, bool there, int lane) {
        ok_k = there;
        if (!there) return;
#pragma unroll
        for (int i = 0; i < kVec; ++i) k[i] = ldg_stream(run + i * 512 + lane * 16);
        const uint8_t *par = run + Kv4<D>::kParamOff;
        kp[0] = __ldg(reinterpret_cast<const uint2 *>(par) + (lane >> 2));
        kp[1] = __ldg(reinterpret_cast<const uint2 *>(par) + (lane >> 2) + 8);
    }
    __device__ __forceinline__ void load_values(const uint8_t *run, bool there, int lane) {
        ok_v = there;
        if (!there) return;
        const uint8_t *par = run + Kv4<D>::kParamOff;
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = ldg_stream(run + Kv4<D>::kValueOff + i * 512 + lane * 16);
        vp[0] = __ldg(reinterpret_cast<const uint4 *>(par) + (lane & 3));
        vp[1] = __ldg(reinterpret_cast<const uint4 *>(par) + (lane & 3) + 4);
    }
    // Keys into the tile at shared address `tile`, what is known of its tokens into `info`; `left`: tokens of the request from the
    // run's first on.  Returns what put_values needs to know: a bit for each token that holds NaN, and kWideRun.
    static constexpr uint32_t kWideRun = 0x10000u;
    __device__ __forceinline__ uint32_t put_keys(uint32_t tile, Info *info, int warp, int left, int lane) const {
        const int r = lane >> 2, c = lane & 3, t0 = warp * 16;
        uint32_t mark = 0u, scaled = 0u;
        bool fits = true;
#pragma unroll
        for (int hi = 0; hi < 2; ++hi) {
            const int t = r + 8 * hi;
            const bool live = ok_k && t < left, nan = live && (not_finite(kp[hi].x) || not_finite(kp[hi].y));
            mark |= ((live ? 1u : 0u) | (nan ? 0x10000u : 0u)) << t;
            const bool use = live && !nan;
            float s = use ? bf16_lo(kp[hi].x) : 0.0f, z = use ? bf16_hi(kp[hi].x) : 0.0f;
            fits = fits && (!use || value_fits(kp[hi].y));
            const float top = use ? largest(kp[hi].x) : 0.0f;
            if (top != 0.0f && !(top >= 0.0625f && top < 32768.0f)) {
                const int ex = min(max((int)(__float_as_uint(top) >> 23), 2), 252);
                const float down = __uint_as_float((uint32_t)(254 - ex) << 23);
                s *= down;
                z *= down;
                scaled |= 1u << t;
                if (c == 0) info->k_mul[t0 + t] = __uint_as_float((uint32_t)ex << 23);
            }
            const Affine a = {twice_f16(s), twice_f16(s * 0.0625f), twice_f16(z)};
            if (D == 128) {
                // the lanes c and c + 2 write to the same banks: the upper two take their words the other way round
                const uint4 u = k[D == 128 ? hi : 0];
                const bool swap = (c & 2) != 0;
                const uint32_t w0 = swap ? u.z : u.x, w1 = swap ? u.w : u.y, w2 = swap ? u.x : u.z, w3 = swap ? u.y : u.w;
                const int p0 = 4 * c + (swap ? 2 : 0), p2 = 4 * c + (swap ? 0 : 2);
                store16(tile + piece_at(t0 + t, p0), values_f16(w0, a));
                store16(tile + piece_at(t0 + t, p0 + 1), values_f16(w1, a));
                store16(tile + piece_at(t0 + t, p2), values_f16(w2, a));
                store16(tile + piece_at(t0 + t, p2 + 1), values_f16(w3, a));
            } else {
                store16(tile + piece_at(t0 + t, 2 * c), values_f16(hi ? k[0].z : k[0].x, a));
                store16(tile + piece_at(t0 + t, 2 * c + 1), values_f16(hi ? k[0].w : k[0].y, a));
            }
        }
        mark = __reduce_or_sync(0xFFFFFFFFu, mark);
        scaled = __reduce_or_sync(0xFFFFFFFFu, scaled);
        fits = __all_sync(0xFFFFFFFFu, fits);
        if (lane == 0) {
            reinterpret_cast<uint16_t *>(info->there)[warp] = (uint16_t)mark;
            reinterpret_cast<uint16_t *>(info->poison)[warp] = (uint16_t)(mark >> 16);
            reinterpret_cast<uint16_t *>(info->scaled)[warp] = (uint16_t)scaled;
            info->wide_runs[warp] = fits ? 0 : 1;
            info->odd[warp] = mark != 0xFFFFu || scaled != 0u || !fits ? 1 : 0;
        }
        return mark >> 16 | (fits ? 0u : kWideRun);
    }
    // `odd`: as put_keys returned it.  Whoever sees a token of NaN gets NaN by its score, so its value is left out whole: a finite one
    // beside a key of NaN was not looked at for whether fp16 holds it.
    __device__ __forceinline__ void put_values(uint32_t tile, int t0, int left, uint32_t odd, int lane) const {
        const bool wide = (odd & kWideRun) != 0u;
        const int r = lane >> 2, c = lane & 3;
#pragma unroll
        for (int hi = 0; hi < 2; ++hi)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int t = 2 * c + e + 8 * hi;
                const uint32_t par = e ? vp[hi].w : vp[hi].y;
                const bool use = ok_v && t < left && !((odd >> t) & 1u);
                float s = use ? bf16_lo(par) : 0.0f, z = use ? bf16_hi(par) : 0.0f;
                uint32_t w0, w1 = 0u;
                if (D == 128) {
                    const uint4 u = v[D == 128 ? hi : 0];
                    w0 = e ? u.z : u.x;
                    w1 = e ? u.w : u.y;
                } else {
                    w0 = hi ? (e ? v[0].w : v[0].z) : (e ? v[0].y : v[0].x);
                }
                const bool swap = D == 128 && (r & 1) != 0;          // as above: odd r the other way round
                const int at = D == 128 ? 2 * r : r;
                if (!wide) {
                    s *= kValueMul;
                    z *= kValueMul;
                    const Affine a = {twice_f16(s), twice_f16(s * 0.0625f), twice_f16(z)};
                    store16(tile + piece_at(t0 + t, at + (swap ? 1 : 0)), values_f16(swap ? w1 : w0, a));
                    if (D == 128) store16(tile + piece_at(t0 + t, at + (swap ? 0 : 1)), values_f16(swap ? w0 : w1, a));
                } else {
                    const Affine a = {twice_bf16(s), 0u, twice_bf16(z)};
                    store16(tile + piece_at(t0 + t, at + (swap ? 1 : 0)), finite_bf16(values_bf16(swap ? w1 : w0, a)));
                    if (D == 128) store16(tile + piece_at(t0 + t, at + (swap ? 0 : 1)), finite_bf16(values_bf16(swap ? w0 : w1, a)));
                }
            }
    }
};

template <int D>
__device__ __forceinline__ void fill_role(const AttnArgs &a, const LineStart &line, Walk &w, uint32_t k_at, uint32_t v_at, Info *info, Bars *bars,
                                          volatile int *dead, int warp, int lane) {
    constexpr uint32_t kTileBytes = D * 2 * kTile;
    const int runs_page = a.page >> 4;
    const long long head_bytes = (long long)runs_page * Kv4<D>::kRunBytes;
    const uint32_t key_full = smem_u32(bars->key_full), key_empty = smem_u32(bars->key_empty);
    const uint32_t val_full = smem_u32(bars->val_full), val_empty = smem_u32(bars->val_empty);
    walk_enter(w, a, line, lane);
    uint32_t n = 0u;                             // tiles filled so far
    while (walk_next(w, a, lane)) {
        const int32_t *table = a.table + (long long)w.rq.b * a.table_stride;
        const uint8_t *head = a.cache + w.h * head_bytes;
        const int step1 = w.step1, kv = w.rq.kv;
        int step = w.step0, id = -1, sub = 0;
        auto lookup = [&](int s) {
            const int run = s * kRunsTile + warp;
            id = -1;
            if (s < step1 && run * 16 < kv) {
                const int blk = run / runs_page;
                id = __ldg(table + blk);
                sub = run - blk * runs_page;
            }
        };
        Fill<D> f;
        const uint8_t *run = head;
        bool there = false;
        auto locate = [&]() {
            there = id >= 0 && id < a.n_blocks;
            run = head + id * (head_bytes * a.Hkv) + (long long)sub * Kv4<D>::kRunBytes;
        };
        const int t0 = warp * 16;
        uint32_t odd_next = 0u;                                    // of the run whose keys were put last
        // keys of tile m, the segment's step s; false: the wait ran out
        auto keys = [&](uint32_t m, int s) {
            const uint32_t st = m & 1u;
            if (!warp_wait(key_empty + 8 * st, ((m >> 1) & 1u) ^ 1u, dead)) return false;
            odd_next = f.put_keys(k_at + st * kTileBytes, info + (m & 3), warp, kv - s * kTile - t0, lane);
            fence_smem();
            __syncwarp();
            if (lane == 0) bar_arrive(key_full + 8 * st);
            return true;
        };
        lookup(step);
        locate();
        f.load_keys(run, there, lane);
        f.load_values(run, there, lane);
        lookup(step + 1);
        if (!keys(n, step)) return;
        locate();
        f.load_keys(run, there, lane);
        lookup(step + 2);
        // Keys stay a tile ahead of the values: the products ask for the scores of up to two tiles on before they are done with
        // a tile's values.  Each load is issued as soon as its registers are free.
#pragma unroll 1
        for (; step < step1; ++step, ++n) {
            const uint8_t *val_run = run;
            const bool val_there = there;
            const uint32_t odd = odd_next;
            if (step + 1 < step1) {
                if (!keys(n + 1, step + 1)) return;
                locate();
                f.load_keys(run, there, lane);
                lookup(step + 3);
            }
            const uint32_t st = n & 1u;
            if (!warp_wait(val_empty + 8 * st, ((n >> 1) & 1u) ^ 1u, dead)) return;
            f.put_values(v_at + st * kTileBytes, t0, kv - step * kTile - t0, odd, lane);
            fence_smem();
            __syncwarp();
            if (lane == 0) bar_arrive(val_full + 8 * st);
            f.load_values(val_run, val_there, lane);
        }
        walk_leave(w, a, lane);
    }
}

// ---------------------------------------------------------------------------------------- products
// One warp for each slot: the steps between two products (waits, commits) of one fall beside the products of the other.  The
// whole warp walks, one lane issues.  A slot's own products are in the order of issue, which is all that its buffers need.
template <int D>
__device__ __forceinline__ void product_role(const AttnArgs &a, const LineStart &line, Walk &w, uint32_t tmem, uint32_t q_at, uint32_t k_at,
                                             uint32_t v_at, Bars *bars, const Info *info, volatile int *dead, uint32_t slot, int lane) {
    constexpr uint32_t kTileBytes = D * 2 * kTile, kBlock = kTile * 128 / 16;
    constexpr uint32_t kScore = kProduct | (uint32_t)(kHalf >> 3) << 17, kOut = kProduct | 1u << 16 | (uint32_t)(D >> 3) << 17;
    const uint32_t key_full = smem_u32(bars->key_full), key_empty = smem_u32(bars->key_empty);
    const uint32_t val_full = smem_u32(bars->val_full), val_empty = smem_u32(bars->val_empty);
    const uint32_t score_full = smem_u32(bars->score_full) + 16 * slot, weight_ready = smem_u32(bars->weight_ready) + 16 * slot;
    const uint32_t out_free = smem_u32(bars->out_free) + 8 * slot;
    const uint64_t q_desc = tile_desc(q_at, 16, 1024), k_desc = tile_desc(k_at, 16, 1024), v_desc = tile_desc(v_at, kTile * 128, 1024);
    const uint32_t s_at = tmem + slot * kTile, o_at = tmem + 2 * kTile + slot * D;
    const uint32_t lead = elected();
    walk_enter(w, a, line, lane);
    uint32_t seg = 0u, tiles = 0u, uses = 0u;
    while (walk_next(w, a, lane)) {
        // the same in every lane, which the compiler shall know
        const uint32_t wide = __shfl_sync(0xFFFFFFFFu, w.wide() ? 1u : 0u, 0), n = __shfl_sync(0xFFFFFFFFu, (uint32_t)(w.step1 - w.step0), 0);
        const uint32_t mine = wide ? n : (n + 1u - slot) >> 1;    // token tiles of this slot
        if (!warp_wait(smem_u32(&bars->query_ready), seg & 1u, dead)) return;
        const uint64_t qa = q_desc + (wide & slot) * (kTileBytes >> 4);
        // item i: half i & 1 of the slot's token tile i >> 1
        auto scores = [&](uint32_t i) {
            const uint32_t buf = i & 1u, t = tiles + (wide ? i >> 1 : 2u * (i >> 1) + slot), st = t & 1u;
            if (buf == 0u && !warp_wait(key_full + 8 * st, (t >> 1) & 1u, dead)) return false;
            fence_after();
            const uint64_t ka = k_desc + st * (kTileBytes >> 4) + buf * (kHalf * 128 / 16);
            const uint32_t d = s_at + buf * kHalf;
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks)
                product_ss(d, qa + (ks >> 2) * kBlock + (ks & 3) * 2, ka + (ks >> 2) * kBlock + (ks & 3) * 2, kScore, ks > 0, lead);
            commit_to(score_full + 8 * buf, lead);
            if (buf) {                                             // a stage is free when both slots have used it, or one twice as much
                commit_to(key_empty + 8 * st, lead);
                if (!wide) commit_to(key_empty + 8 * st, lead);
            }
            return true;
        };
        auto outputs = [&](uint32_t i) {
            const uint32_t buf = i & 1u, t = tiles + (wide ? i >> 1 : 2u * (i >> 1) + slot), st = t & 1u;
            if (buf == 0u && !warp_wait(val_full + 8 * st, (t >> 1) & 1u, dead)) return false;
            if (!warp_wait(weight_ready + 8 * buf, (uses + (i >> 1)) & 1u, dead)) return false;
            fence_after();
            const uint64_t va = v_desc + st * (kTileBytes >> 4) + buf * (kHalf * 128 / 16);
            const uint32_t p = s_at + buf * kHalf;
            const uint32_t odd = __shfl_sync(0xFFFFFFFFu, *reinterpret_cast<const uint32_t *>(&info[t & 3].wide_runs[4 * buf]), 0);
            if (odd == 0u) {
#pragma unroll
                for (int ks = 0; ks < kHalf / 16; ++ks) product_ts(o_at, p + ks * 8, va + ks * 128, kOut, i > 0u || ks > 0, lead);
            } else {                                               // a run of 16 tokens each
#pragma unroll
                for (int ks = 0; ks < kHalf / 16; ++ks)
                    product_ts(o_at, p + ks * 8, va + ks * 128, (odd >> (8 * ks)) & 1u ? kOut | kWithBf16 : kOut, i > 0u || ks > 0, lead);
            }
            commit_to(out_free, lead);
            if (buf) {
                commit_to(val_empty + 8 * st, lead);
                if (!wide) commit_to(val_empty + 8 * st, lead);
            }
            return true;
        };
        const uint32_t items = 2u * mine;
#pragma unroll 1
        for (uint32_t i = 0; i < min(items, 2u); ++i)
            if (!scores(i)) return;
#pragma unroll 1
        for (uint32_t i = 0; i < items; ++i) {
            if (!outputs(i)) return;
            if (i + 2u < items && !scores(i + 2u)) return;
        }
        commit_to(smem_u32(&bars->out_done), lead);
        tiles += n;
        uses += mine;
        ++seg;
        walk_leave(w, a, lane);
    }
}

// ----------------------------------------------------------------------------------------- softmax
__device__ __forceinline__ uint32_t low_bits(int n) { return n <= 0 ? 0u : n >= 32 ? 0xFFFFFFFFu : (1u << n) - 1u; }
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&p);
}

__device__ __forceinline__ uint32_t pack2_f16(float lo, float hi) {
    const __half2 p = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&p);
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float y;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
    return y;
}
__device__ __forceinline__ void fma2(float &x, float &y, float s, float b) {      // both times s plus b
    asm("{\n .reg .b64 v, m, a;\n mov.b64 v, {%0, %1};\n mov.b64 m, {%2, %2};\n mov.b64 a, {%3, %3};\n"
        " fma.rn.f32x2 v, v, m, a;\n mov.b64 {%0, %1}, v;\n}" : "+f"(x), "+f"(y) : "f"(s), "f"(b));
}
__device__ __forceinline__ void add2(float &x, float &y, float a, float b) {
    asm("{\n .reg .b64 v, w;\n mov.b64 v, {%0, %1};\n mov.b64 w, {%2, %3};\n add.rn.f32x2 v, v, w;\n mov.b64 {%0, %1}, v;\n}"
        : "+f"(x), "+f"(y) : "f"(a), "f"(b));
}

template <int D>
__device__ __forceinline__ void softmax_role(const AttnArgs &a, const LineStart &line, Walk &w, uint32_t tmem_all, uint32_t q_at, Bars *bars,
                                             const Info *info, float *s_m, float *s_l, float *s_back, volatile int *dead, int slot, int warp, int lane) {
    constexpr uint32_t kTileBytes = D * 2 * kTile;
    const int me = warp * 32 + lane;                               // row of the slot's tile
    const uint32_t tmem = tmem_all + ((uint32_t)(warp * 32) << 16);
    const uint32_t s_at = tmem + slot * kTile, o_at = tmem + 2 * kTile + slot * D;
    walk_enter(w, a, line, lane);
    uint32_t seg = 0u, used = 0u, freed = 0u, tile_n = 0u;
    while (walk_next(w, a, lane)) {
        const bool wide = w.wide();
        const int step0 = w.step0, n = w.step1 - step0;
        const int row = w.row_first() + (wide ? slot * kTile : 0) + me, qi = row / a.group;
        const bool live = row < w.rq.rows;
        const long long token = w.rq.row0 + qi;
        const int head = w.h * a.group + row - qi * a.group;
        // queries into shared memory (the products of the segment before are done: out_done was waited for); kRowLanes lanes share a
        // row, so that a load takes whole rows and a store all banks
        constexpr int kRowLanes = D / 8, kRowsTurn = 32 / kRowLanes;
        if (wide || slot == 0) {
            const uint32_t q_tile = q_at + slot * kTileBytes;
            const unsigned long long src = (unsigned long long)(a.q + token * a.q_t + (long long)head * a.q_h);
            const uint32_t lives = __ballot_sync(0xFFFFFFFFu, live);
            const int piece = lane % kRowLanes;
            uint4 x[kRowLanes];
#pragma unroll
            for (int i = 0; i < kRowLanes; ++i) {
                const int rr = i * kRowsTurn + lane / kRowLanes;
                const uint4 *from = reinterpret_cast<const uint4 *>(__shfl_sync(0xFFFFFFFFu, src, rr)) + piece;
                x[i] = make_uint4(0u, 0u, 0u, 0u);
                if ((lives >> rr) & 1u) x[i] = __ldg(from);
            }
#pragma unroll
            for (int i = 0; i < kRowLanes; ++i) {
                const int rr = warp * 32 + i * kRowsTurn + lane / kRowLanes;
                // the largest magnitude, as bits (infinities and NaN lie above all numbers, and stay what they are below)
                uint32_t top = __vmaxu2(__vmaxu2(x[i].x & 0x7FFF7FFFu, x[i].y & 0x7FFF7FFFu), __vmaxu2(x[i].z & 0x7FFF7FFFu, x[i].w & 0x7FFF7FFFu));
#pragma unroll
                for (int o = 1; o < kRowLanes; o <<= 1) top = __vmaxu2(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
                top = max(top & 0xFFFFu, top >> 16);
                // the row's largest number to 1 .. 2, with the scale's sign; taken back below
                const int ex = min(max((int)(top >> 7), 27), 227);
                const float up = copysignf(__uint_as_float((uint32_t)(254 - ex) << 23), a.scale_log2);
                const uint32_t v[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
                uint32_t h[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) h[e] = pack2_f16(bf16_lo(v[e]) * up, bf16_hi(v[e]) * up);
                store16(q_tile + piece_at(rr, piece), make_uint4(h[0], h[1], h[2], h[3]));
                if (piece == 0) s_back[slot * kTile + rr] = __uint_as_float((uint32_t)ex << 23);
            }
            fence_smem();
        }
        __syncwarp();
        if (lane == 0) bar_arrive(smem_u32(&bars->query_ready));
        // what a product with the row's queries is multiplied with; a unit of one tile has them from slot 0
        if (!wide) pair_barrier(1, kSoftWarps * 32);
        // (never 0, which would make NaN of the -infinity of what is not seen; the smallest normal number moves nothing)
        const float scale = fmaxf(fabsf(a.scale_log2) * s_back[(wide ? slot * kTile : 0) + me], 1.17549435e-38f);
        const int past = w.rq.kv - w.rq.n_new;
        // rows beyond the unit's see everything: what they hold is not used, and their tiles need no masks
        const int lim = !live ? 0x7FFFFFFF : a.mask_kind == DSP_MASK_CAUSAL ? min(w.rq.kv, past + qi + 1) : w.rq.kv;
        const int all = live && a.mask_kind == DSP_MASK_BITS ? min(past, lim) : lim;      // tokens below are seen without a look at the bits
        const bool some = __any_sync(0xFFFFFFFFu, live);
        const uint32_t *bits = a.bits ? a.bits + token * a.words : nullptr;
        float m = -CUDART_INF_F, l = 0.0f;
        bool fresh = true;                                         // nothing of this slot is in its output yet
        const int halves = 2 * (wide ? n : (n + 1 - slot) >> 1);
#pragma unroll 1
        for (int i = 0; i < halves; ++i) {
            const uint32_t buf = i & 1;
            const uint32_t weight_bar = smem_u32(&bars->weight_ready[slot * 2 + buf]);
            if (!warp_wait(smem_u32(&bars->score_full[slot * 2 + buf]), (used + (i >> 1)) & 1u, dead)) break;
            fence_after();
            if (!some) {                                           // a warp without rows: its part of the tile stays what it is
                if (lane == 0) bar_arrive(weight_bar);
                continue;
            }
            const uint32_t at = s_at + buf * kHalf;
            float x[2][32];
            tmem_load32(at, x[0]);
            tmem_load32(at + 32, x[1]);
            const int tile = wide ? i >> 1 : 2 * (i >> 1) + slot, t0 = (step0 + tile) * kTile + (int)buf * kHalf;
            const Info *inf = info + ((tile_n + tile) & 3);
            const uint32_t odd = *reinterpret_cast<const uint32_t *>(&inf->odd[4 * buf]);
            const bool part = live && (t0 + kHalf > all || odd != 0u);
            tmem_loaded(x[0]);
            tmem_loaded(x[1]);
            if (__any_sync(0xFFFFFFFFu, part)) {                   // at the ends of what a tile's rows see
                const uint2 there = *reinterpret_cast<const uint2 *>(&inf->there[2 * buf]), poison = *reinterpret_cast<const uint2 *>(&inf->poison[2 * buf]);
                const uint2 scaled = *reinterpret_cast<const uint2 *>(&inf->scaled[2 * buf]);
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int u0 = t0 + 32 * k;
                    uint32_t v = low_bits(lim - u0) & (k ? there.y : there.x);
                    if (live && a.mask_kind == DSP_MASK_BITS && u0 + 32 > past && v) {
                        const int j0 = u0 - past;                  // new token that the piece's first place holds
                        const int w0 = j0 >> 5, sh = j0 & 31;
                        const uint32_t lo = w0 >= 0 && w0 < a.words ? __ldg(bits + w0) : w0 < 0 ? 0xFFFFFFFFu : 0u;
                        const uint32_t hi = w0 + 1 >= 0 && w0 + 1 < a.words ? __ldg(bits + w0 + 1) : 0u;
                        v &= sh ? (lo >> sh) | (hi << (32 - sh)) : lo;
                    }
                    const uint32_t nan = v & (k ? poison.y : poison.x), mul = k ? scaled.y : scaled.x;
                    if (mul) {
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if ((mul >> e) & 1u) x[k][e] *= inf->k_mul[kHalf * buf + 32 * k + e];
                    }
#pragma unroll
                    for (int e = 0; e < 32; ++e) x[k][e] = (v >> e) & 1u ? x[k][e] : -CUDART_INF_F;
                    if (nan) {
#pragma unroll
                        for (int e = 0; e < 32; ++e) x[k][e] = (nan >> e) & 1u ? CUDART_NAN_F : x[k][e];
                    }
                }
            }
            // the row's maximum; only where it passes the one so far by 2^8 does that move, and the output with it
            float tops[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int e = 0; e < 32; e += 2) tops[(e >> 1) & 3] = max3(tops[(e >> 1) & 3], x[k][e], x[k][e + 1]);
            const float top = max3(fmaxf(tops[0], tops[1]), tops[2], tops[3]) * scale;
            const bool move = top > m + 8.0f || (m == -CUDART_INF_F && top > m);
            if (__any_sync(0xFFFFFFFFu, move)) {
                const float to = move ? top : m, keep = m == to ? 1.0f : ex2_approx(m - to);
                m = to;
                l *= keep;
                // between the product with the weights before these, which may still be running, and the one with these
                if (!fresh) {
                    if (!warp_wait(smem_u32(&bars->out_free[slot]), (freed + i - 1) & 1u, dead)) break;
                    fence_after();
#pragma unroll 1
                    for (int k = 0; k < D / 8; ++k) {
                        float y[8];
                        tmem_load8(o_at + 8 * k, y);
#pragma unroll
                        for (int e = 0; e < 8; ++e) y[e] *= keep;
                        tmem_store8(o_at + 8 * k, y);
                    }
                }
            }
            fresh = false;
            const float base = m == -CUDART_INF_F ? 0.0f : m - kWeightUp;
            float sums[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int k = 0; k < 2; ++k) {
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    uint32_t p[4];
#pragma unroll
                    for (int e = 0; e < 8; e += 2) {
                        float a0 = x[k][8 * h + e], a1 = x[k][8 * h + e + 1];
                        fma2(a0, a1, scale, -base);
                        a0 = ex2_approx(a0);
                        a1 = ex2_approx(a1);
                        add2(sums[e & 2], sums[(e & 2) + 1], a0, a1);
                        p[e >> 1] = pack2_f16(a0, a1);
                    }
                    tmem_store4(at + 16 * k + 4 * h, p);           // over scores that are in registers
                }
            }
            l += (sums[0] + sums[1]) + (sums[2] + sums[3]);
            if (odd) {                                             // weights of runs whose values are bf16: as bf16 too, with the values' factor
                const uint32_t wide_runs = *reinterpret_cast<const uint32_t *>(&inf->wide_runs[4 * buf]);
                if (wide_runs) tmem_stored();
#pragma unroll 1
                for (int k = 0; k < 4; ++k) {
                    if (!((wide_runs >> (8 * k)) & 1u)) continue;
                    float y[8];
                    uint32_t p[4];
                    tmem_load8(at + 8 * k, y);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const uint32_t both = __float_as_uint(y[e]);
                        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&both));
                        p[e & 3] = pack2(f.x * kValueMul, f.y * kValueMul);
                        if ((e & 3) == 3) tmem_store4(at + 8 * k + e - 3, p);
                    }
                }
            }
            tmem_stored();
            fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(weight_bar);
        }
        used += halves >> 1;
        freed += halves;
        tile_n += n;
        if (!*dead) warp_wait(smem_u32(&bars->out_done), seg & 1u, dead);
        fence_after();
        // a unit of one tile: slot 0 joins both slots' sums; otherwise every slot has its own rows
        float m1 = -CUDART_INF_F, l1 = 0.0f;
        if (!wide) {
            if (slot == 1) {
                s_m[me] = m;
                s_l[me] = l;
            }
            pair_barrier(1, kSoftWarps * 32);
            if (slot == 0) {
                m1 = s_m[me];
                l1 = n > 1 ? s_l[me] : 0.0f;
            }
        }
        if (wide || slot == 0) {
            const bool two = !wide && n > 1;
            const float top = two ? fmaxf(m, m1) : m;
            const float f0 = m == top ? 1.0f : ex2_approx(m - top), f1 = m1 == top ? 1.0f : ex2_approx(m1 - top);
            float sum = two ? fmaf(l1, f1, l * f0) : l;
            if (*dead) sum = CUDART_NAN_F;
            const bool whole = w.step0 == 0 && w.step1 == w.steps;
            const float inv = sum == 0.0f ? 0.0f : whole ? 1.0f / (sum * kValueMul) : 1.0f / kValueMul;
            const int part_row = slot * kTile + me;
            const uint32_t q_tile = q_at + slot * kTileBytes;
            float *part = a.part + ((long long)blockIdx.x * 2 + (w.step0 == 0 ? 1 : 0)) * (2 * kTile * (D + 2));
#pragma unroll 1
            for (int k = 0; k < D / 32; ++k) {
                float x[32];
                tmem_load32(o_at + 32 * k, x);
                if (two) {
                    float y[32];
                    tmem_load32(o_at + D + 32 * k, y);
                    tmem_loaded(x);
                    tmem_loaded(y);
#pragma unroll
                    for (int e = 0; e < 32; ++e) x[e] = fmaf(y[e], f1, x[e] * f0);
                } else {
                    tmem_loaded(x);
                }
                if (*dead) {
#pragma unroll
                    for (int e = 0; e < 32; ++e) x[e] = CUDART_NAN_F;
                }
                if (whole) {                                       // by way of the queries' place, whose products are done
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        store16(q_tile + piece_at(me, 4 * k + e),
                                sum == 0.0f ? make_uint4(0u, 0u, 0u, 0u)
                                            : make_uint4(pack2(x[8 * e] * inv, x[8 * e + 1] * inv), pack2(x[8 * e + 2] * inv, x[8 * e + 3] * inv),
                                                         pack2(x[8 * e + 4] * inv, x[8 * e + 5] * inv), pack2(x[8 * e + 6] * inv, x[8 * e + 7] * inv)));
                } else {                                           // rows lie next to each other, as the lanes do
                    float4 *dst = reinterpret_cast<float4 *>(part) + 8 * k * (2 * kTile) + part_row;
#pragma unroll
                    for (int e = 0; e < 8; ++e) dst[e * (2 * kTile)] = make_float4(x[4 * e] * inv, x[4 * e + 1] * inv, x[4 * e + 2] * inv, x[4 * e + 3] * inv);
                }
            }
            if (whole) {
                const int row2 = w.row_first() + part_row, q2 = row2 / a.group;       // once more: registers are short
                const unsigned long long dst =
                    row2 < w.rq.rows ? (unsigned long long)(a.out + ((long long)(w.rq.row0 + q2) * a.Hq + w.h * a.group + row2 - q2 * a.group) * D) : 0ULL;
                __syncwarp();
#pragma unroll
                for (int i = 0; i < kRowLanes; ++i) {
                    const int rr = i * kRowsTurn + lane / kRowLanes, piece = lane % kRowLanes;
                    uint4 *to = reinterpret_cast<uint4 *>(__shfl_sync(0xFFFFFFFFu, dst, rr));
                    if (to) to[piece] = load16(q_tile + piece_at(warp * 32 + rr, piece));
                }
                __syncwarp();                                      // before the next segment's queries take the place
            }
            if (!whole) {
                part[2 * kTile * D + part_row] = top;
                part[2 * kTile * D + 2 * kTile + part_row] = sum;
                if (w.step0 == 0 && me == 0 && slot == 0) {
                    SplitUnit u;
                    u.b = w.rq.b; u.h = w.h; u.tile = w.tile;
                    u.last_cta = cta_of(w.at - w.off + (long long)w.steps * w.weight + kEnter - 1, w.total, w.ctas);
                    a.split[blockIdx.x] = u;
                }
            }
        }
        fence_before();
        if (!wide) pair_barrier(1, kSoftWarps * 32);              // slot 1's output has been read, its sums too
        ++seg;
        walk_leave(w, a, lane);
    }
}

template <int D>
__global__ void __launch_bounds__(kBlockThreads, 1) attn_block_kernel(const AttnArgs a) {
    constexpr uint32_t kTileBytes = D * 2 * kTile;
    extern __shared__ uint8_t s_raw[];
    __shared__ Bars s_bars;
    __shared__ Info s_info[4];
    __shared__ float s_m[kTile], s_l[kTile], s_back[2 * kTile];
    __shared__ long long s_scan[32];
    __shared__ LineStart s_line;
    __shared__ uint32_t s_tmem;
    __shared__ Walk s_walk[kBlockThreads / 32];
    __shared__ int s_dead;
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const uint32_t base = (smem_u32(s_raw) + 1023u) & ~1023u;
    const uint32_t q_at = base, k_at = base + 2 * kTileBytes, v_at = base + 4 * kTileBytes;
    grid_launch_dependents();                                     // the join's CTAs may come as soon as there is room
    if (threadIdx.x == 0) {
        a.split[blockIdx.x].last_cta = -1;
        s_dead = 0;
        for (int i = 0; i < 2; ++i) {
            bar_init(smem_u32(&s_bars.key_full[i]), kFillWarps);
            bar_init(smem_u32(&s_bars.val_full[i]), kFillWarps);
            bar_init(smem_u32(&s_bars.key_empty[i]), kProductWarps);
            bar_init(smem_u32(&s_bars.val_empty[i]), kProductWarps);
            bar_init(smem_u32(&s_bars.out_free[i]), 1);
        }
        for (int i = 0; i < 4; ++i) {
            bar_init(smem_u32(&s_bars.score_full[i]), 1);
            bar_init(smem_u32(&s_bars.weight_ready[i]), kSoftWarps / 2);
        }
        bar_init(smem_u32(&s_bars.query_ready), kSoftWarps);
        bar_init(smem_u32(&s_bars.out_done), kProductWarps);
        bar_init(smem_u32(&s_bars.ended), kProductWarps);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kSoftWarps + kFillWarps) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" :: "r"(smem_u32(&s_tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        fence_before();
    }
    enter_line<BlockRequest>(a, 0, 0, kWide, s_scan, &s_line);         // ends with a barrier of the CTA
    fence_after();
    const uint32_t tmem = __shfl_sync(0xFFFFFFFFu, s_tmem, 0);
    if (s_line.begin < s_line.end) {
        if (warp < kSoftWarps) {
            softmax_role<D>(a, s_line, s_walk[warp], tmem, q_at, &s_bars, s_info, s_m, s_l, s_back, &s_dead, warp >> 2, warp & 3, lane);
        } else if (warp < kSoftWarps + kFillWarps) {
            fill_role<D>(a, s_line, s_walk[warp], k_at, v_at, s_info, &s_bars, &s_dead, warp - kSoftWarps, lane);
        } else {
            product_role<D>(a, s_line, s_walk[warp], tmem, q_at, k_at, v_at, &s_bars, s_info, &s_dead, (uint32_t)(warp - kSoftWarps - kFillWarps), lane);
        }
    }
    __syncwarp();
    // by the lane that issued them: where a wait ran out, products may still be under way, which read this CTA's memory
    if (warp >= kSoftWarps + kFillWarps) commit_to(smem_u32(&s_bars.ended), elected());
    fence_before();
    __syncthreads();
    if (warp == kSoftWarps + kFillWarps) {
        const long long t0 = clock64();
        while (!bar_test(smem_u32(&s_bars.ended), 0u) && clock64() - t0 < kWaitClocks) {}
        __syncwarp();
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" :: "r"(tmem) : "memory");
    }
}

// Joins the partial results of one unit: 16 rows per CTA of 256 threads, the parts of a turn loaded together (by ordinary loads: they
// are written while this kernel's CTAs already wait).
constexpr int kJoinThreads = 256, kJoinTurn = 4, kJoinRows = 16;
template <int D>
__global__ void __launch_bounds__(kJoinThreads) attn_block_join_kernel(const AttnArgs a) {
    grid_dependency_wait();
    constexpr int kPart = 2 * kTile * (D + 2), kChunks = 2 * kTile / kJoinRows, kVec = kJoinRows * (D / 4) / kJoinThreads;
    const int first = blockIdx.x / kChunks, chunk = blockIdx.x % kChunks;
    const SplitUnit u = a.split[first];
    if (u.last_cta < 0) return;
    const int n = u.last_cta - first + 1;
    BlockRequest rq;
    rq.load(a, u.b, 0, 0);
    const int rows = rq.rows_of(u.tile);
    if (chunk * kJoinRows >= rows) return;
    const float *base = a.part + (long long)first * 2 * kPart;
    // a warp takes four rows and eight pieces of four channels: whole sectors of the parts, where rows are neighbours, and of the output
    auto row_of = [&](int i) { return chunk * kJoinRows + ((i >> 5) & 3) * 4 + (i & 3); };
    auto piece_of = [&](int i) { return (i >> 7) * 8 + ((i >> 2) & 7); };
    auto part_of = [&](int i) { return base + (long long)(2 * i + (i == 0 ? 1 : 0)) * kPart; };
    float4 x[kVec];
    float m[kVec], l[kVec];
#pragma unroll
    for (int k = 0; k < kVec; ++k) {
        x[k] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        m[k] = -CUDART_INF_F;
        l[k] = 0.0f;
    }
    for (int i0 = 0; i0 < n; i0 += kJoinTurn) {
#pragma unroll
        for (int k = 0; k < kVec; ++k) {
            const int i = threadIdx.x + k * kJoinThreads, row = row_of(i), piece = piece_of(i);
            float4 y[kJoinTurn];
            float my[kJoinTurn], ly[kJoinTurn];
#pragma unroll
            for (int w = 0; w < kJoinTurn; ++w) {
                const bool ok = i0 + w < n && row < rows;
                const float *p = part_of(i0 + w);
                my[w] = ok ? p[2 * kTile * D + row] : -CUDART_INF_F;
                ly[w] = ok ? p[2 * kTile * D + 2 * kTile + row] : 0.0f;
                y[w] = ok ? reinterpret_cast<const float4 *>(p)[piece * (2 * kTile) + row] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            }
            float top = m[k];
#pragma unroll
            for (int w = 0; w < kJoinTurn; ++w) top = fmaxf(top, my[w]);
            const float keep = m[k] == top ? 1.0f : ex2_approx(m[k] - top);
            m[k] = top;
            x[k].x *= keep; x[k].y *= keep; x[k].z *= keep; x[k].w *= keep;
            l[k] *= keep;
#pragma unroll
            for (int w = 0; w < kJoinTurn; ++w) {
                const float f = my[w] == top ? 1.0f : ex2_approx(my[w] - top);
                x[k].x = fmaf(y[w].x, f, x[k].x); x[k].y = fmaf(y[w].y, f, x[k].y);
                x[k].z = fmaf(y[w].z, f, x[k].z); x[k].w = fmaf(y[w].w, f, x[k].w);
                l[k] = fmaf(ly[w], f, l[k]);
            }
        }
    }
#pragma unroll
    for (int k = 0; k < kVec; ++k) {
        const int i = threadIdx.x + k * kJoinThreads, row = row_of(i), ch = piece_of(i) * 4;
        if (row >= rows) continue;
        const float inv = 1.0f / l[k];
        const int rr = u.tile * 2 * kTile + row, qi = rr / a.group;
        *reinterpret_cast<uint2 *>(a.out + ((long long)(rq.row0 + qi) * a.Hq + u.h * a.group + rr - qi * a.group) * D + ch) =
            l[k] == 0.0f ? make_uint2(0u, 0u) : make_uint2(pack2(x[k].x * inv, x[k].y * inv), pack2(x[k].z * inv, x[k].w * inv));
    }
}

template <int D>
cudaError_t launch(const AttnArgs &a, int grid, cudaStream_t st) {
    constexpr int smem = 6 * D * 2 * kTile + 1024;
    static std::atomic<unsigned long long> done{0};
    cudaError_t e = allow_shared(attn_block_kernel<D>, smem, done);
    if (e != cudaSuccess) return e;
    attn_block_kernel<D><<<grid, kBlockThreads, smem, st>>>(a);
    e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    return launch_dependent(attn_block_join_kernel<D>, (unsigned)grid * (2 * kTile / kJoinRows), kJoinThreads, 0, st, a, true);
}

}  // namespace

size_t attn_block_part_bytes(int D) { return (size_t)2 * kTile * (D + 2) * sizeof(float); }

cudaError_t attn_block_launch(const AttnArgs &a, int D, int grid, cudaStream_t st) {
    return D == 64 ? launch<64>(a, grid, st) : launch<128>(a, grid, st);
}

}  // namespace dsp
