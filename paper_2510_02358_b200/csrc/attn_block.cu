// The kernel of dsp_attn_kv4 for many query rows (verified blocks and trees times the heads of a group,
// prompts): bound by the tensor cores.
//
// One CTA per SM.  A unit is up to 256 query rows of one key head against a stretch of the cache; its
// rows are two tiles of 128 that share every key and value tile, or, with at most 128 rows, one tile
// whose even and odd token tiles go to the two halves of the CTA.  Either way there are two slots, each
// with 128 x 128 scores and a 128 x D output in tensor memory (512 columns together), so that the tensor
// cores work on one slot while the other's scores are exponentiated.
//
//   warps 0-7   softmax, four per slot, one thread per query row: maximum, exponentials, weights in bf16
//               back into the scores' columns as the second product's operand
//   warps 8-15  the tiles' codes (four warps keys, four values): 16-byte loads one tile ahead in
//               registers, four bits to bf16 values, swizzled stores; two stages of each
//   warp 16     one thread issues the products: S = Q K^T, O += P V
//
// Here a cached number is expanded once for 128 or 256 rows, so it becomes a whole bf16 value on the way
// (code * scale + offset, one rounding): folding the scales into the sums, as the kernel for few rows
// does, would cost each score more than that.
//
// The running maximum moves only when a row's scores pass it by 2^8, and only then is the output in
// tensor memory rescaled (by the softmax warps, between two products of their slot).
//
// Tokens that nobody may see (beyond the length, of a missing block) become zeros, and those whose scale
// or offset is NaN too, with a bit beside the tile: the rows that see such a token get a NaN score.
#include "attn.cuh"
#include "attn_block.h"

namespace dsp {
namespace {

constexpr int kSoftWarps = 8, kFillWarps = 8, kBlockThreads = (kSoftWarps + kFillWarps + 1) * 32;
constexpr int kTile = 128;                       // query rows of a slot, tokens of a tile
constexpr int kRunsTile = kTile / 16;
constexpr long long kWaitClocks = 4000000000LL;  // about two seconds: a wait that long has failed

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
__device__ __forceinline__ void commit_to(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(bar) : "memory");
}
// Operand tiles lie in shared memory as blocks of 64 channels: [block][row][128 bytes], the 16-byte
// pieces of a row exchanged by its number modulo 8 (the 128-byte swizzle).  The same bytes serve as an
// operand contracted over the channels (queries, keys) and as one contracted over the rows (values).
__device__ __forceinline__ uint64_t tile_desc(uint32_t addr, uint32_t lead_bytes, uint32_t stride_bytes) {
    return (uint64_t)((addr & 0x3FFFF) >> 4) | (uint64_t)(lead_bytes >> 4) << 16 | (uint64_t)(stride_bytes >> 4) << 32 |
           (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
constexpr uint32_t kBf16Product = 1u << 4 | 1u << 7 | 1u << 10 | (uint32_t)(kTile >> 4) << 24;      // fp32 sums, bf16 operands, 128 rows
__device__ __forceinline__ void product_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
                 :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void product_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
                 :: "r"(d), "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
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
__device__ __forceinline__ void tmem_store32(uint32_t at, const float (&x)[32]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
                 "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
                 :: "r"(at), "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]),
                    "f"(x[8]), "f"(x[9]), "f"(x[10]), "f"(x[11]), "f"(x[12]), "f"(x[13]), "f"(x[14]), "f"(x[15]),
                    "f"(x[16]), "f"(x[17]), "f"(x[18]), "f"(x[19]), "f"(x[20]), "f"(x[21]), "f"(x[22]), "f"(x[23]),
                    "f"(x[24]), "f"(x[25]), "f"(x[26]), "f"(x[27]), "f"(x[28]), "f"(x[29]), "f"(x[30]), "f"(x[31]) : "memory");
}
__device__ __forceinline__ void tmem_store16(uint32_t at, const uint32_t (&x)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
                 :: "r"(at), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7]),
                    "r"(x[8]), "r"(x[9]), "r"(x[10]), "r"(x[11]), "r"(x[12]), "r"(x[13]), "r"(x[14]), "r"(x[15]) : "memory");
}
// The registers pass through the wait, so that nothing uses them before it.
__device__ __forceinline__ void tmem_loaded(float (&x)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(x[0]), "+f"(x[1]), "+f"(x[2]), "+f"(x[3]), "+f"(x[4]), "+f"(x[5]), "+f"(x[6]), "+f"(x[7]),
                   "+f"(x[8]), "+f"(x[9]), "+f"(x[10]), "+f"(x[11]), "+f"(x[12]), "+f"(x[13]), "+f"(x[14]), "+f"(x[15]),
                   "+f"(x[16]), "+f"(x[17]), "+f"(x[18]), "+f"(x[19]), "+f"(x[20]), "+f"(x[21]), "+f"(x[22]), "+f"(x[23]),
                   "+f"(x[24]), "+f"(x[25]), "+f"(x[26]), "+f"(x[27]), "+f"(x[28]), "+f"(x[29]) , "+f"(x[30]), "+f"(x[31]) :: "memory");
}
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void pair_barrier(int id, int threads) { asm volatile("bar.sync %0, %1;" :: "r"(id), "r"(threads) : "memory"); }

// ------------------------------------------------------------------------------- cut of the work
// A request's units: tiles of 256 rows, for each tile its key heads.  Lengths are counted in tile
// products (128 rows x 128 tokens): 2 for each token tile of a unit with more than 128 rows, else 1.
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
    __device__ __forceinline__ int weight(int tile) const { return rows_of(tile) > kTile ? 2 : 1; }
    __device__ __forceinline__ int steps(int tile) const {
        const int last = (tile * 2 * kTile + rows_of(tile) - 1) / group;
        const int end = causal ? min(kv, kv - n_new + last + 1) : kv;
        return max(1, (end + kTile - 1) / kTile);
    }
    __device__ __forceinline__ long long length(int Hkv) const {
        if (!causal) {
            const long long whole = rows / (2 * kTile), rest = rows - whole * 2 * kTile, n = max(1, (kv + kTile - 1) / kTile);
            return Hkv * n * (2 * whole + (rest > kTile ? 2 : rest > 0 ? 1 : 0));
        }
        long long n = 0;
        for (int t = 0; t < tiles; ++t) n += (long long)steps(t) * weight(t);
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
            const long long len = (long long)rq.steps(tile) * rq.weight(tile) * a.Hkv;
            if (rest < len) break;
            rest -= len;
            ++tile;
        }
        const int unit = rq.steps(tile) * rq.weight(tile);
        h = (int)(rest / unit);
        off = (int)(rest - (long long)h * unit);
    }
    // The next segment; false at the share's end.
    __device__ __forceinline__ bool next(const AttnArgs &a) {
        while (at < end) {
            steps = rq.steps(tile);
            weight = rq.weight(tile);
            const int len = steps * weight, take = (int)min((long long)(len - off), end - at);
            step0 = off / weight;
            step1 = off + take == len ? steps : (off + take) / weight;
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
    __device__ __forceinline__ bool wide() const { return weight == 2; }
    __device__ __forceinline__ int row_first() const { return tile * 2 * kTile; }
};

struct Bars {
    uint64_t key_full[2], key_empty[2], val_full[2], val_empty[2], score_full[2], weight_ready[2], query_ready, out_done;
};
struct Info {                                    // beside a token tile, one bit per token
    uint32_t there[4], poison[4];
};

// ------------------------------------------------------------------------------- codes to values
__device__ __forceinline__ uint32_t biased_pair(uint32_t w, int i) {
    uint32_t y;
    asm("lop3.b32 %0, %1, 0x000F000F, 0x43004300, 0xEA;" : "=r"(y) : "r"(w >> (4 * i)));
    return y;
}
// Eight channels: (128 + code) - 128 is exact, then code * s + z is rounded once.
__device__ __forceinline__ uint4 values8(uint32_t w, uint32_t s2, uint32_t z2) {
    uint32_t v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t code;
        asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(code) : "r"(biased_pair(w, i)), "r"(0x43004300u));
        asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(v[i]) : "r"(code), "r"(s2), "r"(z2));
    }
    return make_uint4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void store16(uint32_t at, const uint4 &v) {
    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" :: "r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ uint32_t both_lo(uint32_t p) { return __byte_perm(p, p, 0x1010); }
__device__ __forceinline__ uint32_t both_hi(uint32_t p) { return __byte_perm(p, p, 0x3232); }
__device__ __forceinline__ bool not_finite(uint32_t p) { return (p & 0x7FFFu) >= 0x7F80u || (p & 0x7FFF0000u) >= 0x7F800000u; }
// Where the 16-byte piece `piece` (channels 8 piece ..) of row t lies in an operand tile.
__device__ __forceinline__ uint32_t piece_at(int t, int piece) {
    return (uint32_t)((piece >> 3) * (kTile * 128) + t * 128 + (((piece & 7) ^ (t & 7)) << 4));
}

// One fill warp's two runs of a tile, keys or values.
template <int D, bool kKeys> struct Fill {
    static constexpr int kVec = D / 64;
    uint4 v[2][kVec];
    uint4 p[2][2];                               // keys: {.xy} of the tokens r and r + 8; values: tokens 2c, 2c+1 and 2c+8, 2c+9
    bool ok[2];
    __device__ __forceinline__ void load(const AttnArgs &a, const Walk &w, int step, int warp, const int (&id)[2], const int (&sub)[2],
                                         long long head_bytes, int lane) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            ok[x] = id[x] >= 0 && id[x] < a.n_blocks;
            if (!ok[x]) continue;
            const uint8_t *run = a.cache + ((long long)id[x] * a.Hkv + w.h) * head_bytes + (long long)sub[x] * Kv4<D>::kRunBytes;
#pragma unroll
            for (int i = 0; i < kVec; ++i) v[x][i] = ldg_stream(run + (kKeys ? 0 : Kv4<D>::kValueOff) + i * 512 + lane * 16);
            const uint8_t *par = run + Kv4<D>::kParamOff;
            if (kKeys) {
                const uint2 lo = __ldg(reinterpret_cast<const uint2 *>(par) + (lane >> 2)), hi = __ldg(reinterpret_cast<const uint2 *>(par) + (lane >> 2) + 8);
                p[x][0] = make_uint4(lo.x, lo.y, 0u, 0u);
                p[x][1] = make_uint4(hi.x, hi.y, 0u, 0u);
            } else {
                p[x][0] = __ldg(reinterpret_cast<const uint4 *>(par) + (lane & 3));
                p[x][1] = __ldg(reinterpret_cast<const uint4 *>(par) + (lane & 3) + 4);
            }
        }
    }
    // Into the tile at shared address `tile`; token0: place of the tile's first token in the request, kv: its length.
    __device__ __forceinline__ void put(uint32_t tile, Info *info, int token0, int kv, int warp, int lane) const {
        const int r = lane >> 2, c = lane & 3;
        uint32_t there = 0u, poison = 0u;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int t0 = (warp * 2 + x) * 16;
            if (kKeys) {
#pragma unroll
                for (int hi = 0; hi < 2; ++hi) {
                    const int t = t0 + r + 8 * hi;
                    const bool live = ok[x] && token0 + t < kv, nan = live && (not_finite(p[x][hi].x) || not_finite(p[x][hi].y));
                    there |= (live ? 1u : 0u) << (t & 31);
                    poison |= (nan ? 1u : 0u) << (t & 31);
                    const bool use = live && !nan;
                    const uint32_t s2 = use ? both_lo(p[x][hi].x) : 0u, z2 = use ? both_hi(p[x][hi].x) : 0u;
                    if (D == 128) {
                        // the lanes c and c + 2 write to the same banks: the upper two take their words the other way round
                        const uint4 u = v[x][D == 128 ? hi : 0];
                        const bool swap = (c & 2) != 0;
                        const uint32_t w0 = swap ? u.z : u.x, w1 = swap ? u.w : u.y, w2 = swap ? u.x : u.z, w3 = swap ? u.y : u.w;
                        const int p0 = 4 * c + (swap ? 2 : 0), p2 = 4 * c + (swap ? 0 : 2);
                        store16(tile + piece_at(t, p0), values8(w0, s2, z2));
                        store16(tile + piece_at(t, p0 + 1), values8(w1, s2, z2));
                        store16(tile + piece_at(t, p2), values8(w2, s2, z2));
                        store16(tile + piece_at(t, p2 + 1), values8(w3, s2, z2));
                    } else {
                        const uint4 u = v[x][0];
                        store16(tile + piece_at(t, 2 * c), values8(hi ? u.z : u.x, s2, z2));
                        store16(tile + piece_at(t, 2 * c + 1), values8(hi ? u.w : u.y, s2, z2));
                    }
                }
            } else {
#pragma unroll
                for (int hi = 0; hi < 2; ++hi)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int t = t0 + 2 * c + e + 8 * hi;
                        const uint32_t par = e ? p[x][hi].w : p[x][hi].y;
                        const bool use = ok[x] && token0 + t < kv && !not_finite(par);
                        const uint32_t s2 = use ? both_lo(par) : 0u, z2 = use ? both_hi(par) : 0u;
                        if (D == 128) {
                            const uint4 u = v[x][D == 128 ? hi : 0];
                            const uint32_t a0 = e ? u.z : u.x, a1 = e ? u.w : u.y;
                            const bool swap = (r & 1) != 0;              // as above: odd r the other way round
                            store16(tile + piece_at(t, 2 * r + (swap ? 1 : 0)), values8(swap ? a1 : a0, s2, z2));
                            store16(tile + piece_at(t, 2 * r + (swap ? 0 : 1)), values8(swap ? a0 : a1, s2, z2));
                        } else {
                            const uint4 u = v[x][0];
                            store16(tile + piece_at(t, r), values8(hi ? (e ? u.w : u.z) : (e ? u.y : u.x), s2, z2));
                        }
                    }
            }
        }
        if (kKeys) {
            there = __reduce_or_sync(0xFFFFFFFFu, there);
            poison = __reduce_or_sync(0xFFFFFFFFu, poison);
            if (lane == 0) {
                info->there[warp] = there;
                info->poison[warp] = poison;
            }
        }
    }
};

template <int D, bool kKeys>
__device__ __forceinline__ void fill_role(const AttnArgs &a, const LineStart &line, uint32_t tiles, Info *info, const uint32_t (&full)[2],
                                          const uint32_t (&empty)[2], volatile int *dead, int warp, int lane) {
    const int runs_page = a.page >> 4;
    const long long head_bytes = (long long)runs_page * Kv4<D>::kRunBytes;
    Walk w;
    w.enter(a, line);
    uint32_t n = 0u;                             // tiles filled so far
    while (w.next(a)) {
        const int32_t *table = a.table + (long long)w.rq.b * a.table_stride;
        const int last_run = (w.rq.kv + 15) >> 4;
        int id[2], sub[2];
        auto lookup = [&](int step) {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int run = step * kRunsTile + warp * 2 + x;
                id[x] = -1;
                sub[x] = 0;
                if (step < w.step1 && run < last_run) {
                    const int blk = run / runs_page;
                    id[x] = __ldg(table + blk);
                    sub[x] = run - blk * runs_page;
                }
            }
        };
        Fill<D, kKeys> f;
        lookup(w.step0);
        f.load(a, w, w.step0, warp, id, sub, head_bytes, lane);
        lookup(w.step0 + 1);
        for (int step = w.step0; step < w.step1; ++step, ++n) {
            const Fill<D, kKeys> cur = f;
            if (step + 1 < w.step1) f.load(a, w, step + 1, warp, id, sub, head_bytes, lane);
            lookup(step + 2);
            const int st = n & 1;
            if (!warp_wait(empty[st], ((n >> 1) & 1) ^ 1u, dead)) return;
            cur.put(tiles + st * (D * 2 * kTile), info + (n & 3), step * kTile, w.rq.kv, warp, lane);
            fence_smem();
            __syncwarp();
            if (lane == 0) bar_arrive(full[st]);
        }
        w.leave(a);
    }
}

// ---------------------------------------------------------------------------------------- products
template <int D>
__device__ __forceinline__ void product_role(const AttnArgs &a, const LineStart &line, uint32_t tmem, uint32_t q_at, uint32_t k_at, uint32_t v_at,
                                             Bars *bars, volatile int *dead) {
    constexpr uint32_t kTileBytes = D * 2 * kTile;
    constexpr uint32_t kScore = kBf16Product | (uint32_t)(kTile >> 3) << 17, kOut = kBf16Product | 1u << 16 | (uint32_t)(D >> 3) << 17;
    Walk w;
    w.enter(a, line);
    uint32_t seg = 0u, keys = 0u, vals = 0u, used[2] = {0u, 0u};
    while (w.next(a)) {
        const bool wide = w.wide();
        const int n = (w.step1 - w.step0) * (wide ? 2 : 1);
        if (!bar_wait(smem_u32(&bars->query_ready), seg & 1u, dead)) return;
        uint32_t key_have = 0u, val_have = 0u;   // tiles of this segment that have been waited for
        bool fine = true;
        auto scores = [&](int i) {
            const int slot = i & 1;
            const uint32_t t = (uint32_t)(wide ? i >> 1 : i), st = (keys + t) & 1u;
            if (key_have <= t) {
                fine = fine && bar_wait(smem_u32(&bars->key_full[st]), ((keys + t) >> 1) & 1u, dead);
                key_have = t + 1;
                if (!fine) return;
            }
            fence_after();
            const uint32_t qa = q_at + (wide ? slot : 0) * kTileBytes, ka = k_at + st * kTileBytes;
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
                const uint32_t by = (uint32_t)((ks >> 2) * (kTile * 128) + (ks & 3) * 32);
                product_ss(tmem + slot * kTile, tile_desc(qa + by, 16, 1024), tile_desc(ka + by, 16, 1024), kScore, ks > 0);
            }
            if (!wide || slot == 1) commit_to(smem_u32(&bars->key_empty[st]));
            commit_to(smem_u32(&bars->score_full[slot]));
        };
        auto outputs = [&](int i) {
            const int slot = i & 1;
            const uint32_t t = (uint32_t)(wide ? i >> 1 : i), st = (vals + t) & 1u;
            fine = fine && bar_wait(smem_u32(&bars->weight_ready[slot]), used[slot] & 1u, dead);
            ++used[slot];
            if (fine && val_have <= t) {
                fine = bar_wait(smem_u32(&bars->val_full[st]), ((vals + t) >> 1) & 1u, dead);
                val_have = t + 1;
            }
            if (!fine) return;
            fence_after();
            const uint32_t va = v_at + st * kTileBytes;
#pragma unroll
            for (int ks = 0; ks < kTile / 16; ++ks)
                product_ts(tmem + 2 * kTile + slot * D, tmem + slot * kTile + ks * 8, tile_desc(va + ks * 2048, kTile * 128, 1024), kOut,
                           i > 1 || ks > 0);
            if (!wide || slot == 1) commit_to(smem_u32(&bars->val_empty[st]));
        };
        scores(0);
        if (n > 1 && fine) scores(1);
        for (int i = 0; i < n && fine; ++i) {
            outputs(i);
            if (i + 2 < n && fine) scores(i + 2);
        }
        if (!fine) return;
        commit_to(smem_u32(&bars->out_done));
        keys += w.step1 - w.step0;
        vals += w.step1 - w.step0;
        ++seg;
        w.leave(a);
    }
}

// ----------------------------------------------------------------------------------------- softmax
__device__ __forceinline__ uint32_t low_bits(int n) { return n <= 0 ? 0u : n >= 32 ? 0xFFFFFFFFu : (1u << n) - 1u; }
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&p);
}

template <int D>
__device__ __forceinline__ void softmax_role(const AttnArgs &a, const LineStart &line, uint32_t tmem_all, uint32_t q_at, Bars *bars, const Info *info,
                                             float *s_m, float *s_l, volatile int *dead, int slot, int warp, int lane) {
    constexpr uint32_t kTileBytes = D * 2 * kTile;
    const int me = warp * 32 + lane;                               // row of the slot's tile
    const uint32_t tmem = tmem_all + ((uint32_t)(warp * 32) << 16);
    const uint32_t s_at = tmem + slot * kTile, o_at = tmem + 2 * kTile + slot * D;
    const float scale = fabsf(a.scale_log2);
    Walk w;
    w.enter(a, line);
    uint32_t seg = 0u, used = 0u, tile_n = 0u;
    while (w.next(a)) {
        const bool wide = w.wide();
        const int n = w.step1 - w.step0;
        const int row = w.row_first() + (wide ? slot * kTile : 0) + me, qi = row / a.group;
        const bool live = row < w.rq.rows;
        const long long token = w.rq.row0 + qi;
        const int head = w.h * a.group + row - qi * a.group;
        // queries into shared memory (the products of the segment before are done: out_done was waited for)
        if (wide || slot == 0) {
            const uint32_t dst = q_at + (wide ? slot : 0) * kTileBytes;
            const uint32_t flip = a.scale_log2 < 0.0f ? 0x80008000u : 0u;      // the scale's sign goes into the queries
            const uint4 *src = reinterpret_cast<const uint4 *>(a.q + token * a.q_t + (long long)head * a.q_h);
#pragma unroll
            for (int i = 0; i < D / 8; ++i) {
                uint4 x = make_uint4(0u, 0u, 0u, 0u);
                if (live) x = __ldg(src + i);
                x.x ^= flip; x.y ^= flip; x.z ^= flip; x.w ^= flip;
                store16(dst + piece_at(me, i), x);
            }
            fence_smem();
        }
        __syncwarp();
        if (lane == 0) bar_arrive(smem_u32(&bars->query_ready));
        const int past = w.rq.kv - w.rq.n_new;
        const int lim = !live ? 0 : a.mask_kind == DSP_MASK_CAUSAL ? min(w.rq.kv, past + qi + 1) : w.rq.kv;
        const int all = a.mask_kind == DSP_MASK_BITS ? min(past, lim) : lim;      // tokens below are seen without a look at the bits
        const uint32_t *bits = a.bits ? a.bits + token * a.words : nullptr;
        float m = -CUDART_INF_F, l = 0.0f;
        bool fresh = true;                                         // nothing of this slot is in its output yet
        for (int i = wide ? 0 : slot; i < n; i += wide ? 1 : 2) {
            if (*dead) break;
            if (!warp_wait(smem_u32(&bars->score_full[slot]), used & 1u, dead)) break;
            ++used;
            fence_after();
            const int t0 = (w.step0 + i) * kTile;
            const Info *inf = info + ((tile_n + i) & 3);
            uint32_t hole = 0u;
#pragma unroll
            for (int k = 0; k < 4; ++k) hole |= ~inf->there[k] | inf->poison[k];
            const bool part = __any_sync(0xFFFFFFFFu, hole != 0u || t0 + kTile > all);
            // tokens of piece k (32 of them) that this row sees, and those of them that hold NaN
            auto seen = [&](int k) {
                const int u0 = t0 + 32 * k;
                uint32_t v = low_bits(lim - u0) & inf->there[k];
                if (a.mask_kind == DSP_MASK_BITS && u0 + 32 > past && v) {
                    const int j0 = u0 - past;                      // new token that the piece's first place holds
                    const int w0 = j0 >> 5, sh = j0 & 31;
                    const uint32_t lo = w0 >= 0 && w0 < a.words ? __ldg(bits + w0) : w0 < 0 ? 0xFFFFFFFFu : 0u;
                    const uint32_t hi = w0 + 1 >= 0 && w0 + 1 < a.words ? __ldg(bits + w0 + 1) : 0u;
                    v &= sh ? (lo >> sh) | (hi << (32 - sh)) : lo;
                }
                return v;
            };
            float x[32], top = -CUDART_INF_F;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                tmem_load32(s_at + 32 * k, x);
                tmem_loaded(x);
                if (part) {
                    const uint32_t v = seen(k);
#pragma unroll
                    for (int e = 0; e < 32; ++e) x[e] = (v >> e) & 1u ? x[e] : -CUDART_INF_F;
                }
#pragma unroll
                for (int e = 0; e < 32; ++e) top = fmaxf(top, x[e]);
            }
            top *= scale;                                          // scale >= 0; 0 * -inf is NaN, which the next line takes for "no move"
            bool move = top > (fresh ? -CUDART_INF_F : m + 8.0f) && top > m;
            if (scale == 0.0f) move = fresh && m != 0.0f;
            if (__any_sync(0xFFFFFFFFu, move)) {
                const float to = move ? (scale == 0.0f ? 0.0f : top) : m;
                const float keep = m == to ? 1.0f : ex2_approx(m - to);
                m = to;
                l *= keep;
                if (!fresh) {
#pragma unroll 1
                    for (int k = 0; k < D / 32; ++k) {
                        tmem_load32(o_at + 32 * k, x);
                        tmem_loaded(x);
#pragma unroll
                        for (int e = 0; e < 32; ++e) x[e] *= keep;
                        tmem_store32(o_at + 32 * k, x);
                    }
                }
            }
            fresh = false;
            const float base = m == -CUDART_INF_F ? 0.0f : m;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                tmem_load32(s_at + 32 * k, x);
                tmem_loaded(x);
                if (part) {
                    const uint32_t v = seen(k), nan = v & inf->poison[k];
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        float y = ex2_approx(fmaf(x[e], scale, -base));
                        y = (v >> e) & 1u ? y : 0.0f;
                        x[e] = (nan >> e) & 1u ? CUDART_NAN_F : y;
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 32; ++e) x[e] = ex2_approx(fmaf(x[e], scale, -base));
                }
                uint32_t p[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    l += x[2 * e];
                    l += x[2 * e + 1];
                    p[e] = pack2(x[2 * e], x[2 * e + 1]);
                }
                tmem_store16(s_at + 16 * k, p);
            }
            tmem_stored();
            fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(smem_u32(&bars->weight_ready[slot]));
        }
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
            const float inv = sum == 0.0f ? 0.0f : whole ? 1.0f / sum : 1.0f;
            const int part_row = (wide ? slot * kTile : 0) + me;
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
                if (!live) continue;
                if (whole) {
                    uint4 *dst = reinterpret_cast<uint4 *>(a.out + (token * a.Hq + head) * D + 32 * k);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        dst[e] = sum == 0.0f ? make_uint4(0u, 0u, 0u, 0u)
                                             : make_uint4(pack2(x[8 * e] * inv, x[8 * e + 1] * inv), pack2(x[8 * e + 2] * inv, x[8 * e + 3] * inv),
                                                          pack2(x[8 * e + 4] * inv, x[8 * e + 5] * inv), pack2(x[8 * e + 6] * inv, x[8 * e + 7] * inv));
                } else {
                    float4 *dst = reinterpret_cast<float4 *>(part + (long long)part_row * D + 32 * k);
#pragma unroll
                    for (int e = 0; e < 8; ++e) dst[e] = make_float4(x[4 * e], x[4 * e + 1], x[4 * e + 2], x[4 * e + 3]);
                }
            }
            if (!whole) {
                part[2 * kTile * D + part_row] = top;
                part[2 * kTile * D + 2 * kTile + part_row] = sum;
                if (w.step0 == 0 && me == 0 && slot == 0) {
                    SplitUnit u;
                    u.b = w.rq.b; u.h = w.h; u.tile = w.tile;
                    u.last_cta = cta_of(w.at - w.off + (long long)w.steps * w.weight - 1, w.total, w.ctas);
                    a.split[blockIdx.x] = u;
                }
            }
        }
        fence_before();
        if (!wide) pair_barrier(1, kSoftWarps * 32);              // slot 1's output has been read, its sums too
        ++seg;
        w.leave(a);
    }
}

template <int D>
__global__ void __launch_bounds__(kBlockThreads, 1) attn_block_kernel(const AttnArgs a) {
    constexpr uint32_t kTileBytes = D * 2 * kTile;
    extern __shared__ uint8_t s_raw[];
    __shared__ Bars s_bars;
    __shared__ Info s_info[4];
    __shared__ float s_m[kTile], s_l[kTile];
    __shared__ long long s_scan[32];
    __shared__ LineStart s_line;
    __shared__ uint32_t s_tmem;
    __shared__ int s_dead;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t base = (smem_u32(s_raw) + 1023u) & ~1023u;
    const uint32_t q_at = base, k_at = base + 2 * kTileBytes, v_at = base + 4 * kTileBytes;
    if (threadIdx.x == 0) {
        a.split[blockIdx.x].last_cta = -1;
        s_dead = 0;
        for (int i = 0; i < 2; ++i) {
            bar_init(smem_u32(&s_bars.key_full[i]), kFillWarps / 2);
            bar_init(smem_u32(&s_bars.val_full[i]), kFillWarps / 2);
            bar_init(smem_u32(&s_bars.key_empty[i]), 1);
            bar_init(smem_u32(&s_bars.val_empty[i]), 1);
            bar_init(smem_u32(&s_bars.score_full[i]), 1);
            bar_init(smem_u32(&s_bars.weight_ready[i]), kSoftWarps / 2);
        }
        bar_init(smem_u32(&s_bars.query_ready), kSoftWarps);
        bar_init(smem_u32(&s_bars.out_done), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kSoftWarps + kFillWarps) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" :: "r"(smem_u32(&s_tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        fence_before();
    }
    enter_line<BlockRequest>(a, 0, 0, 2, s_scan, &s_line);         // ends with a barrier of the CTA
    fence_after();
    const uint32_t tmem = s_tmem;
    if (s_line.begin < s_line.end) {
        if (warp < kSoftWarps) {
            softmax_role<D>(a, s_line, tmem, q_at, &s_bars, s_info, s_m, s_l, &s_dead, warp >> 2, warp & 3, lane);
        } else if (warp < kSoftWarps + kFillWarps) {
            const int f = warp - kSoftWarps;
            if (f < kFillWarps / 2) {
                const uint32_t full[2] = {smem_u32(&s_bars.key_full[0]), smem_u32(&s_bars.key_full[1])};
                const uint32_t empty[2] = {smem_u32(&s_bars.key_empty[0]), smem_u32(&s_bars.key_empty[1])};
                fill_role<D, true>(a, s_line, k_at, s_info, full, empty, &s_dead, f, lane);
            } else {
                const uint32_t full[2] = {smem_u32(&s_bars.val_full[0]), smem_u32(&s_bars.val_full[1])};
                const uint32_t empty[2] = {smem_u32(&s_bars.val_empty[0]), smem_u32(&s_bars.val_empty[1])};
                fill_role<D, false>(a, s_line, v_at, s_info, full, empty, &s_dead, f - kFillWarps / 2, lane);
            }
        } else if (lane == 0) {
            product_role<D>(a, s_line, tmem, q_at, k_at, v_at, &s_bars, &s_dead);
        }
    }
    __syncwarp();
    fence_before();
    __syncthreads();
    if (warp == kSoftWarps + kFillWarps) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" :: "r"(tmem) : "memory");
    }
}

// Joins the partial results of one unit, 16 rows per CTA of 128 threads.
template <int D>
__global__ void __launch_bounds__(128) attn_block_join_kernel(const AttnArgs a) {
    grid_dependency_wait();
    constexpr int kPart = 2 * kTile * (D + 2), kChunks = 2 * kTile / 16;
    const int first = blockIdx.x / kChunks, chunk = blockIdx.x % kChunks;
    const SplitUnit u = a.split[first];
    if (u.last_cta < 0) return;
    const int n = u.last_cta - first + 1;
    BlockRequest rq;
    rq.load(a, u.b, 0, 0);
    const int rows = rq.rows_of(u.tile);
    auto part_of = [&](int i) { return a.part + ((long long)(first + i) * 2 + (i == 0 ? 1 : 0)) * kPart; };
    for (int i = threadIdx.x; i < 16 * (D / 4); i += 128) {
        const int row = chunk * 16 + i / (D / 4), ch = (i % (D / 4)) * 4;
        if (row >= rows) continue;
        float top = -CUDART_INF_F, sum = 0.0f;
        float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int w = 0; w < n; ++w) top = fmaxf(top, part_of(w)[2 * kTile * D + row]);
        for (int w = 0; w < n; ++w) {
            const float *p = part_of(w);
            const float m = p[2 * kTile * D + row], f = m == top ? 1.0f : ex2_approx(m - top);
            const float4 y = *reinterpret_cast<const float4 *>(p + (long long)row * D + ch);
            x.x = fmaf(y.x, f, x.x); x.y = fmaf(y.y, f, x.y); x.z = fmaf(y.z, f, x.z); x.w = fmaf(y.w, f, x.w);
            sum = fmaf(p[2 * kTile * D + 2 * kTile + row], f, sum);
        }
        const float inv = 1.0f / sum;
        const int rr = u.tile * 2 * kTile + row, qi = rr / a.group;
        *reinterpret_cast<uint2 *>(a.out + ((long long)(rq.row0 + qi) * a.Hq + u.h * a.group + rr - qi * a.group) * D + ch) =
            sum == 0.0f ? make_uint2(0u, 0u) : make_uint2(pack2(x.x * inv, x.y * inv), pack2(x.z * inv, x.w * inv));
    }
}

template <int D>
cudaError_t launch(const AttnArgs &a, int grid, cudaStream_t st) {
    constexpr int smem = 6 * D * 2 * kTile + 1024;
    cudaError_t e = cudaFuncSetAttribute(attn_block_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    attn_block_kernel<D><<<grid, kBlockThreads, smem, st>>>(a);
    e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    return launch_dependent(attn_block_join_kernel<D>, (unsigned)grid * (2 * kTile / 16), 128, 0, st, a, true);
}

}  // namespace

size_t attn_block_part_bytes(int D) { return (size_t)2 * kTile * (D + 2) * sizeof(float); }

cudaError_t attn_block_launch(const AttnArgs &a, int D, int grid, cudaStream_t st) {
    return D == 64 ? launch<64>(a, grid, st) : launch<128>(a, grid, st);
}

}  // namespace dsp
