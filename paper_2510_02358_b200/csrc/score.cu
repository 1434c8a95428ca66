// dsp_token_logprobs: log-probabilities of given tokens, entropy, rank and the best alternatives of every row.
//
// One pass over the logits by the row engine (stream_core.cuh, row_engine.cuh): slices stream through shared memory, the CTA that is
// through with a row last finishes it.  Its own parts are the sums at a temperature (TokenPass::sums), the rank of the first token
// (TokenPass::count) and rows that start or end inside a 16-byte piece: the whole pieces between are streamed, and what lies outside of
// them (fewer than two pieces, one element a lane) joins the result when the row is finished, so an odd vocabulary costs nothing.
//
// The rank needs one comparison per logit and no index: a token that precedes token t in the vocabulary comes before it with an equal
// logit, a later one does not, so pieces before t's count what exceeds the next smaller number and the others what exceeds t's logit.
// It is looked for only in tiles whose largest logit reaches the token's.
//
// The floor is one read of the rows.  Measured (device time): 2048 rows of 152064 bf16 of which 25% are not read, 84 us = 5.5 TB/s, 0.86 of a
// plain copy's rate; 272 rows with 20 alternatives 30 us (0.34: the selection, by one CTA a row, is 7 of them, the rest is that 272 rows are less than
// two waves); 2048 rows of 32003 fp32, 26% not read, nine tokens a row, 44 us (0.68: a row is six tiles, and while one warp finishes it the CTA's ring is
// empty; with three CTAs an SM 17 of 24 warps were active, 38% of the issue slots and 26% of the exponential unit taken).  CTAs that stay and take row
// after row measured 50 us there and 94 on the first: rows that are not read leave some of them idle.
#include <string.h>

#include "dsp_internal.h"
#include "row_engine.cuh"

namespace dsp {
namespace {

struct ScoreArgs {
    const void *logits;
    int B, L, V;
    long long stride_b, stride_l;
    const int32_t *row_len, *tokens;
    int G, K;
    double inv_t, inv_s;      // 1 / T, and back from exponents: 1 / (s T)
    float s;                  // log2(e) / T in 32 bits: all exponents are multiples of it
    uint32_t low;             // the lowest logit that counts, as a word of the logits' type (twice for bf16)
    float low_s;              // and its exponent
    float *logp;
    int32_t *rank, *top_id;
    float *top_logit, *top_logp, *lse, *entropy;
    uint32_t *row_status;
    int inner;                // elements of a row that are streamed: a multiple of a piece's
    int nslices, ntiles_row, nstages;
    RowScratch rs;
    unsigned *rank_acc;       // [rows] zeroed per call
    bool own_status;          // a row is all of its status word: written, else OR-ed into
};

// The number just below x (NaN below -inf: everything exceeds it).
__device__ __forceinline__ uint32_t below_bits(float x) {
    const uint32_t b = __float_as_uint(x);
    if (x == 0.f) return 0x80000001u;
    if (b == 0xFF800000u) return 0x7FFFFFFFu;
    return (b & 0x80000000u) ? b + 1u : b - 1u;
}
__device__ __forceinline__ uint32_t below_bits_bf16(float x) {
    const uint32_t b = __float_as_uint(x) >> 16;
    if (x == 0.f) return 0x8001u;
    if (b == 0xFF80u) return 0x7FFFu;
    return (b & 0x8000u) ? b + 1u : b - 1u;
}

template <typename DT>
struct TokenPass {
    static constexpr bool kOwnTile = true;
    const DT *row;            // the whole row
    const int32_t *tokens;    // the row's tokens
    int G;
    bool ranked;
    unsigned *acc;
    float s;
    uint32_t low;             // what masked logits are raised to in the sums, as a word of DT
    int V, head, inner;
    // rank
    int tok = -1, vec = 0;    // token, and the streamed piece it lies in (pieces: beyond, 0: before)
    bool apart = false;       // it lies in the streamed part: taken out of the sums, score_row adds it
    float xt = 0.f;
    uint32_t ge = 0u, gt = 0u;
    int n = 0;
    // what the row's finish needs of the row, loaded by the first warp while the row streams: a token a lane, the elements outside of
    // the streamed pieces, the piece of the first token
    int mine = -1;
    float x_mine = 0.f, x_outer = 0.f, x_piece = 0.f;

    // the outer element of a lane (lanes 16 and up), -1: none
    __device__ __forceinline__ int outer_at(int lane) const {
        const int i = lane - 16;
        return i < 0 || i >= V - inner ? -1 : i < head ? i : inner + i;
    }
    __device__ __forceinline__ void begin() {
        constexpr int N = Elem<DT>::N;
        const int lane = threadIdx.x;
        if (lane < 32) {
            if (lane < G) mine = tokens[lane];
            if (mine >= 0 && mine < V) x_mine = Elem<DT>::load1(row + mine);
            const int v = outer_at(lane);
            x_outer = v >= 0 ? Elem<DT>::load1(row + v) : -CUDART_INF_F;
        }
        tok = G > 0 ? tokens[0] : -1;            // kept out of the sums with a rank and without
        if (tok < 0 || tok >= V) { tok = -1; xt = CUDART_INF_F; ge = gt = N == 8 ? 0x7F807F80u : 0x7F800000u; return; }   // above everything
        xt = Elem<DT>::load1(row + tok);
        vec = tok < head ? 0 : min((tok - head) / N, inner / N);
        if constexpr (N == 8) {
            gt = (__float_as_uint(xt) >> 16) * 0x10001u;
            ge = below_bits_bf16(xt) * 0x10001u;
        } else {
            gt = __float_as_uint(xt);
            ge = below_bits(xt);
        }
        apart = tok >= head && tok < head + inner;
        if (lane < N && apart) x_piece = Elem<DT>::load1(row + head + vec * N + lane);
    }
    // Logits of a tile that come before the token: looked for only where the tile's largest reaches it.
    __device__ __forceinline__ void count(const uint4 (&v)[kVpt], int base) {
        constexpr int N = Elem<DT>::N;
        const int v0 = base / N + (int)threadIdx.x;
        if constexpr (N == 8) {
            __nv_bfloat162 sum = __floats2bfloat162_rn(0.f, 0.f);          // at most 4 kVpt a half: exact
#pragma unroll
            for (int j = 0; j < kVpt; ++j) {
                const uint32_t w = v0 + j * kThreads < vec ? ge : gt;
                const uint32_t q[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
#pragma unroll
                for (int i = 0; i < 4; ++i) sum = __hadd2(sum, __hgtu2(as_bf162(q[i]), as_bf162(w)));
            }
            n += (int)(__low2float(sum) + __high2float(sum));
        } else {
#pragma unroll
            for (int j = 0; j < kVpt; ++j) {
                const float lim = __uint_as_float(v0 + j * kThreads < vec ? ge : gt);
#pragma unroll
                for (int e = 0; e < N; ++e) n += Elem<DT>::get(v[j], e) <= lim ? 0 : 1;
            }
        }
    }
    // Element e of a piece becomes -inf.
    static __device__ __forceinline__ void hide(uint4 &v, int e) {
        const int at = Elem<DT>::N == 8 ? e >> 1 : e;
        const uint32_t mask = Elem<DT>::N == 4 ? 0xFFFFFFFFu : e & 1 ? 0xFFFF0000u : 0x0000FFFFu;
        const uint32_t word = (Elem<DT>::N == 8 ? 0xFF80FF80u : 0xFF800000u) & mask;
        if (at == 0) v.x = (v.x & ~mask) | word;
        if (at == 1) v.y = (v.y & ~mask) | word;
        if (at == 2) v.z = (v.z & ~mask) | word;
        if (at == 3) v.w = (v.w & ~mask) | word;
    }
    static __device__ __forceinline__ __nv_bfloat162 as_bf162(uint32_t w) { return *reinterpret_cast<const __nv_bfloat162 *>(&w); }
    static __device__ __forceinline__ uint32_t word(__nv_bfloat162 v) { return *reinterpret_cast<const uint32_t *>(&v); }
    static __device__ __forceinline__ float max_of(const uint4 (&v)[kVpt]) {
        if constexpr (Elem<DT>::N == 8) {
            __nv_bfloat162 m[kVpt];
#pragma unroll
            for (int j = 0; j < kVpt; ++j)
                m[j] = __hmax2_nan(__hmax2_nan(as_bf162(v[j].x), as_bf162(v[j].y)), __hmax2_nan(as_bf162(v[j].z), as_bf162(v[j].w)));
#pragma unroll
            for (int j = 1; j < kVpt; ++j) m[0] = __hmax2_nan(m[0], m[j]);
            return max2_nan(bf16_lo(word(m[0])), bf16_hi(word(m[0])));
        } else {
            float m = __uint_as_float(v[0].x);
#pragma unroll
            for (int j = 0; j < kVpt; ++j) {
                m = max3_nan(m, __uint_as_float(v[j].x), __uint_as_float(v[j].y));
                m = max3_nan(m, __uint_as_float(v[j].z), __uint_as_float(v[j].w));
            }
            return m;
        }
    }
    // One tile's share of a thread: S = sum 2^a and T = sum 2^a a over the exponents a = x s - c.  A masked logit counts as `low`: its
    // power is 0, and so is the product (0 * -inf is not).  The first token is left out: next to a token that holds nearly all of the mass an fp32
    // sum has no room for the others, which are all that its log-probability and the entropy are made of then.
    template <bool RAGGED>
    __device__ __forceinline__ float tile(const uint4 (&t)[kVpt], int nvec, int tid, int base, float &c, unsigned long long &S2,
                                          unsigned long long &T2) {
        constexpr int N = Elem<DT>::N;
        uint4 v[kVpt];
#pragma unroll
        for (int j = 0; j < kVpt; ++j) v[j] = t[j];
        const float tm = max_of(v);
        if (!(tm < xt)) {
            count(v, base);
            const int at = vec - base / N - tid;
            if (apart && at >= 0 && at % kThreads == 0) {
#pragma unroll
                for (int j = 0; j < kVpt; ++j)
                    if (at == j * kThreads) hide(v[j], (tok - head) % N);
            }
        }
        const float ts = fmaxf(tm, N == 8 ? bf16_hi(low) : __uint_as_float(low)) * s;
        if (ts > c) {
            const float d = c - ts;
            const float sc = ex2_approx(d);
            const unsigned long long sc2 = pack2(sc, sc);
            T2 = mul2(fma2(S2, pack2(d, d), T2), sc2);
            S2 = mul2(S2, sc2);
            c = ts;
        }
        const unsigned long long nc2 = pack2(-c, -c), s2 = pack2(s, s);
#pragma unroll
        for (int j = 0; j < kVpt; ++j) {
            if (RAGGED && j * kThreads + tid >= nvec) continue;
            const uint32_t q[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
#pragma unroll
            for (int i = 0; i < 4; i += N == 8 ? 1 : 2) {
                float x0, x1;
                if constexpr (N == 8) {
                    const uint32_t w = word(__hmax2_nan(as_bf162(q[i]), as_bf162(low)));
                    x0 = bf16_lo(w);
                    x1 = bf16_hi(w);
                } else {
                    x0 = max2_nan(__uint_as_float(q[i]), __uint_as_float(low));
                    x1 = max2_nan(__uint_as_float(q[i + 1]), __uint_as_float(low));
                }
                const unsigned long long a2 = fma2(pack2(x0, x1), s2, nc2);
                float a0, a1;
                unpack2(a2, a0, a1);
                const unsigned long long e2 = pack2(ex2_approx(a0), ex2_approx(a1));
                S2 = add2(S2, e2);
                T2 = fma2(e2, a2, T2);
            }
        }
        return tm;
    }
    // The slice's count, after the preparation has ended and before the row's ticket.
    __device__ __forceinline__ void hand_in() {
        if (!ranked) return;
        const int all = (int)__reduce_add_sync(0xFFFFFFFFu, (unsigned)n);
        if ((threadIdx.x & 31) == 0 && all) atomicAdd(acc, (unsigned)all);
    }
};

// A row that is not read.
__device__ void score_nothing(const ScoreArgs &a, long long row, int lane) {
    if (a.own_status && lane == 0) a.row_status[row] = 0u;
    for (int i = lane; i < a.G; i += 32) a.logp[row * a.G + i] = -CUDART_INF_F;
    if (lane < a.K) {
        a.top_id[row * a.K + lane] = -1;
        a.top_logit[row * a.K + lane] = -CUDART_INF_F;
        a.top_logp[row * a.K + lane] = -CUDART_INF_F;
    }
    if (lane == 0) {
        if (a.rank) a.rank[row] = -1;
        a.lse[row] = -CUDART_INF_F;
        if (a.entropy) a.entropy[row] = 0.f;
    }
}

// The logit that a lane adds to the sums by itself: one outside of the streamed pieces, the first token (lane 31), or none (-inf).
template <typename DT>
__device__ __forceinline__ float apart_of(const TokenPass<DT> &pass, int lane) {
    static_assert(2 * Elem<DT>::N <= 16, "fewer than 15 outer elements: lane 31 is free");
    return lane == 31 && pass.apart ? pass.xt : pass.x_outer;
}
// The sums of a row from its n partials and those logits, by one warp.
template <typename DT, typename At>
__device__ __forceinline__ void merge_row(const ScoreArgs &a, const TokenPass<DT> &pass, At at, int n, int lane, RowResult &r) {
    const int last = n <= 16 ? 0 : (n + 31) / 32 * 32;   // a lane's last entry is its own logit (up to 16 partials leave room in one round)
    const double e = (double)apart_of(pass, lane) * (double)a.s;
    const float ce = (float)e;
    const double res = (e - (double)ce) * kLn2;          // below 2^-16: 2^res is 1 + res + res^2 / 2 to 2^-50
    WarpPartial own;
    own.S = ce > kRefFloor ? 1.0 + res + 0.5 * res * res : 0.0;
    own.c = ce; own.T = own.S * (e - (double)ce); own.pad = 0;
    if (!(own.S > 0.0)) { own.S = own.T = 0.0; own.c = kRefFloor; }
    WarpPartial none;
    none.S = none.T = 0.0; none.c = kRefFloor; none.pad = 0;
    warp_merge_partials([&](int i) { return i < n ? at(i) : i >= last ? own : none; }, last + 32, lane, r.c, r.S, r.T);
}

// The finish of a row by one warp: the first token and the elements outside of the streamed pieces join (joined: the sums have them), and everything is
// written (counted: of the streamed logits, how many come before the first token; trouble: status bits so far).
template <typename DT>
__device__ void score_row(const ScoreArgs &a, long long row, int b, const DT *rowp, int head, const TokenPass<DT> &pass, RowResult r,
                          bool joined, unsigned counted, uint32_t trouble, int lane) {
    constexpr int N = Elem<DT>::N;
    // one element a lane: before the streamed pieces, then behind them
    const int extra = a.V - a.inner;
    const int v = pass.outer_at(lane);
    const float x = pass.x_outer;
    bool bad = __any_sync(0xFFFFFFFFu, !(x < CUDART_INF_F)) || r.nonfinite;
    unsigned long long key = lane < a.K && r.key ? r.key - (unsigned)head : 0ull;      // ids count from the streamed part
    double c = r.c, S = r.S, T = r.T;
    if (extra > 0) key = merge_top32(key, sort32_desc(x > -CUDART_INF_F ? make_key(x, v) : 0ull, lane), lane);
    if (!joined && (extra > 0 || pass.apart)) {
        const float y = apart_of(pass, lane);
        const double e = (double)y * (double)a.s;
        const float cm = fmaxf(S != 0.0 ? r.c : kRefFloor, warp_max((float)e > kRefFloor ? (float)e : kRefFloor));
        const double d = c - (double)cm, w = S != 0.0 ? exp2(d) : 0.0;
        const double p = y > -CUDART_INF_F ? exp2(e - (double)cm) : 0.0;
        const double S1 = warp_sum(p), T1 = warp_sum(p != 0.0 ? p * (e - (double)cm) : 0.0);
        T = (S != 0.0 ? (T + S * d) * w : 0.0) + T1;
        S = S * w + S1;
        c = cm;
    }
    bad |= !(S > 0.0) || !(S < CUDART_INF) || !(T == T) || !(c > (double)a.low_s) || !(c < CUDART_INF);
    const double log_s = log2(S);
    const double lse = bad ? CUDART_NAN : c * a.inv_s + kLn2 * log_s;
    for (int i = lane; i < a.G; i += 32) {
        const int t = i < 32 ? pass.mine : a.tokens[row * a.G + i];
        const bool in = t >= 0 && t < a.V;
        const float xi = !in || i < 32 ? pass.x_mine : Elem<DT>::load1(rowp + t);
        a.logp[row * a.G + i] = in ? (float)((double)xi * a.inv_t - lse) : -CUDART_INF_F;
    }
    if (lane < a.K) {
        const bool some = key != 0ull;
        const float xv = some ? key_value(key) : -CUDART_INF_F;
        a.top_id[row * a.K + lane] = some ? key_id(key) : -1;
        a.top_logit[row * a.K + lane] = xv;
        a.top_logp[row * a.K + lane] = some ? (float)((double)xv * a.inv_t - lse) : -CUDART_INF_F;
    }
    if (a.rank) {
        int rank = -1;
        if (pass.tok >= 0) {
            // before the token: of the outer elements, and of its own piece (counted without equals)
            int n = v >= 0 && (x > pass.xt || (x == pass.xt && v < pass.tok)) ? 1 : 0;
            const int u = head + pass.vec * N + lane;
            if (pass.tok >= head && pass.tok < head + a.inner && lane < N && u < pass.tok && pass.x_piece == pass.xt) ++n;
            rank = (int)(__reduce_add_sync(0xFFFFFFFFu, (unsigned)n) + counted);
        }
        if (lane == 0) a.rank[row] = rank;
    }
    if (lane == 0) {
        a.lse[row] = (float)lse;
        if (a.entropy) a.entropy[row] = bad ? CUDART_NAN_F : (float)(kLn2 * log_s - T / S * a.inv_s);
        if (bad) trouble |= DSP_ROW_NONFINITE_INPUT;
        if (a.own_status) a.row_status[b] = trouble;
        else if (trouble) atomicOr(&a.row_status[b], trouble);
    }
}

// The sums of a row whose best tokens nobody asks for: as row_engine, without the selection.  True in warp 0 of the CTA that is through last.
template <typename DT>
__device__ bool score_sums(const ScoreArgs &a, const DT *inner, long long row, int slice, int b, StreamBars &bars, unsigned char *ring,
                           TokenPass<DT> &pass, RowResult &r) {
    __shared__ int s_last;
    const int tid = threadIdx.x, lane = tid & 31, warp = warp_index();
    int s0, s1;
    slice_range<DT>(slice, a.nslices, a.ntiles_row, a.inner, s0, s1);
    ColTop top;
    ColSums cs;
    stream_slice<DT, true>(inner, s0, s1, a.nstages, bars, ring, top, cs, pass);
    if (!(top.seen < CUDART_INF_F)) cs.S = CUDART_NAN_F;         // NaN or +inf: the row's sum says so
    const WarpPartial p = warp_partial(cs);
    grid_dependency_wait();
    pass.hand_in();
    if (lane == 0) {
        if (a.nslices > 1) {
            a.rs.wpart[(row * a.nslices + slice) * kWarps + warp] = p;
            __threadfence();
        } else {
            bars.wp[warp] = p;
        }
    }
    __syncthreads();
    if (tid == 0) {
        if (bars.timed_out) atomicOr(&a.row_status[b], (unsigned)DSP_ROW_TIMEOUT);
        s_last = a.nslices == 1 || atomicAdd(&a.rs.row_ticket[row], 1u) == (unsigned)a.nslices - 1;
    }
    if (warp != 0) return false;
    __syncwarp();
    if (!s_last) return false;
    if (a.nslices > 1) {
        __threadfence();
        const WarpPartial *wp = a.rs.wpart + row * a.nslices * kWarps;
        merge_row(a, pass, [&](int i) {
            WarpPartial q;
            q.S = __ldcg(&wp[i].S); q.T = __ldcg(&wp[i].T); q.c = __ldcg(&wp[i].c); q.pad = 0;
            return q;
        }, a.nslices * kWarps, lane, r);
    } else {
        merge_row(a, pass, [&](int i) { return bars.wp[i]; }, kWarps, lane, r);
    }
    r.key = 0ull;
    r.nonfinite = false;
    return true;
}

// CTAS: of an SM.
template <typename DT, int CTAS>
__global__ void __launch_bounds__(kThreads, CTAS) score_kernel(const ScoreArgs a) {
    constexpr int N = Elem<DT>::N;
    extern __shared__ __align__(128) unsigned char ring[];
    __shared__ StreamBars bars;
    const unsigned row32 = blockIdx.x / (unsigned)a.nslices;
    const long long row = row32;
    const int slice = (int)(blockIdx.x - row32 * (unsigned)a.nslices);
    const int b = (int)(row32 / (unsigned)a.L), l = (int)(row32 - (unsigned)b * (unsigned)a.L), lane = threadIdx.x & 31;
    if (a.row_len && l >= a.row_len[b]) {                // whole CTA alike
        if (slice == 0 && threadIdx.x < 32) score_nothing(a, row, lane);
        grid_dependency_wait();                          // a call may have no other row: what follows it has to find the preparation ended
        return;
    }
    const DT *rowp = reinterpret_cast<const DT *>(a.logits) + b * a.stride_b + l * a.stride_l;
    const int head = a.inner == a.V ? 0 : (int)((N - (reinterpret_cast<uintptr_t>(rowp) / sizeof(DT)) % N) % N);
    TokenPass<DT> pass;
    pass.row = rowp;
    pass.tokens = a.tokens + row * a.G;
    pass.G = a.G;
    pass.ranked = a.rank != nullptr;
    pass.acc = a.rank_acc + row;
    pass.s = a.s; pass.low = a.low;
    pass.V = a.V; pass.head = a.inner ? head : 0; pass.inner = a.inner;
    RowResult r;
    if (a.inner && a.K == 0) {
        stream_begin(bars, a.nstages);
        if (!score_sums<DT>(a, rowp + head, row, slice, b, bars, ring, pass, r)) return;
    } else if (a.inner) {
        stream_begin(bars, a.nstages);
        if (!row_engine<DT>(rowp + head, a.inner, a.K, true, row, slice, a.nslices, a.ntiles_row, a.nstages, a.rs,
                            &a.row_status[b], bars, ring, r, pass))
            return;
    } else {                                             // a row shorter than two pieces: one element a lane
        if (threadIdx.x >= 32) return;
        pass.begin();
        grid_dependency_wait();
        r.key = 0ull; r.c = kRefFloor; r.S = 0.0; r.T = 0.0; r.nonfinite = false;
    }
    const unsigned counted = pass.ranked && pass.tok >= 0 && a.inner && lane == 0 ? atomicAdd(pass.acc, 0u) : 0u;
    score_row<DT>(a, row, b, rowp, pass.head, pass, r, a.inner && a.K == 0, counted, 0u, lane);
}

// ---- few rows: the CTAs of a row are a cluster and hand what they found to the first one, which finishes the row; no tickets, so nothing
// has to be prepared where a status word belongs to one row ----
constexpr int kMaxCluster = 8;
constexpr int kClusterTiles = 4;             // tiles of a CTA, all in its ring at once
constexpr int kFinishArea = kFinishBytes + kMaxCluster * kThreads * 8;
struct HandIn {                              // in the first CTA
    uint64_t got;                            // its barrier
    __align__(8) WarpPartial wp[kMaxCluster * kWarps];     // pad: the warp's count of logits before the first token, its top bit a wait that ran out
};
// Stores into the first CTA that are counted, in bytes, by a barrier there: no fence is needed on either side.
__device__ __forceinline__ void send_counted(uint32_t addr, uint32_t bar, unsigned long long v) {
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.b64 [%0], %1, [%2];" ::"r"(addr), "l"(v), "r"(bar) : "memory");
}

template <typename DT>
__global__ void __launch_bounds__(kThreads, 2) score_cluster_kernel(const ScoreArgs a) {
    constexpr int N = Elem<DT>::N;
    extern __shared__ __align__(128) unsigned char ring[];
    __shared__ StreamBars bars;
    __shared__ HandIn hand;
    const unsigned C = (unsigned)a.nslices, row32 = blockIdx.x / C, rank = cluster_rank();
    const long long row = row32;
    const int tid = threadIdx.x, lane = tid & 31, warp = warp_index();
    const int b = (int)(row32 / (unsigned)a.L), l = (int)(row32 - (unsigned)b * (unsigned)a.L);
    if (a.row_len && l >= a.row_len[b]) {                // the whole cluster alike
        if (rank == 0 && warp == 0) score_nothing(a, row, lane);
        grid_dependency_wait();                          // as in score_kernel
        return;
    }
    const DT *rowp = reinterpret_cast<const DT *>(a.logits) + b * a.stride_b + l * a.stride_l;
    const int head = a.inner == a.V ? 0 : (int)((N - (reinterpret_cast<uintptr_t>(rowp) / sizeof(DT)) % N) % N);
    TokenPass<DT> pass;
    pass.row = rowp;
    pass.tokens = a.tokens + row * a.G;
    pass.G = a.G;
    pass.ranked = a.rank != nullptr;
    pass.acc = nullptr;
    pass.s = a.s; pass.low = a.low;
    pass.V = a.V; pass.head = head; pass.inner = a.inner;
    if (tid == 0) {                                      // before stream_begin's fence and barrier
        mbar_init(&hand.got, 1);
        mbar_expect_tx(&hand.got, C * (kWarps * (unsigned)sizeof(WarpPartial) + (a.K ? kThreads * 8u : 0u)));
    }
    stream_begin(bars, a.nstages);
    cluster_arrive_empty();
    int s0, s1;
    slice_range<DT>((int)rank, (int)C, a.ntiles_row, a.inner, s0, s1);
    ColTop top;
    ColSums cs;
    stream_slice<DT, true>(rowp + head, s0, s1, a.nstages, bars, ring, top, cs, pass);
    if (a.K == 0 && !(top.seen < CUDART_INF_F)) cs.S = CUDART_NAN_F;      // NaN or +inf: the row's sum says so
    const WarpPartial p = warp_partial(cs);
    const unsigned counted = __reduce_add_sync(0xFFFFFFFFu, (unsigned)pass.n);
    unsigned char *area = ring + a.nstages * kTileBytes;
    cluster_wait();                                      // the first CTA is there
    const uint32_t bar = at_rank(&hand.got, 0);
    if (a.K) {
        const uint2 col = pack_col(top);
        send_counted(at_rank(area + kFinishBytes + (rank * kThreads + tid) * 8, 0), bar, (unsigned long long)col.y << 32 | col.x);
    }
    if (lane == 0) {
        const uint32_t to = at_rank(&hand.wp[rank * kWarps + warp], 0);
        const unsigned late = *static_cast<volatile int *>(&bars.timed_out) ? 0x80000000u : 0u;       // the warp saw its own waits run out
        send_counted(to, bar, (unsigned long long)__double_as_longlong(p.S));
        send_counted(to + 8, bar, (unsigned long long)__double_as_longlong(p.T));
        send_counted(to + 16, bar, (unsigned long long)(counted | late) << 32 | __float_as_uint(p.c));
    }
    if (rank != 0) return;
    volatile int never = 0;                              // twice as long as a CTA waits for its copies: what it sends arrives here before this one leaves
    const bool there = mbar_wait(&hand.got, 0u, &never) || mbar_wait(&hand.got, 0u, &never);
    unsigned trouble = __syncthreads_or(!there) ? (unsigned)DSP_ROW_TIMEOUT : 0u;
    RowResult r;
    if (a.K) {
        if (!row_finish<DT>(rowp + head, a.inner, a.K, true, row, (int)C, a.ntiles_row, a.rs, hand.wp, area, r)) return;
    } else {
        if (warp != 0) return;
        merge_row(a, pass, [&](int i) { return hand.wp[i]; }, (int)C * kWarps, lane, r);
        r.key = 0ull;
        r.nonfinite = false;
    }
    unsigned before = 0u, late = 0u;
    for (unsigned i = lane; i < C * kWarps; i += 32) {
        before += (unsigned)hand.wp[i].pad & 0x7FFFFFFFu;
        late |= (unsigned)hand.wp[i].pad >> 31;
    }
    before = __reduce_add_sync(0xFFFFFFFFu, before);
    if (__any_sync(0xFFFFFFFFu, late != 0u)) trouble = DSP_ROW_TIMEOUT;
    grid_dependency_wait();                              // status words that several rows share are zeroed
    score_row<DT>(a, row, b, rowp, head, pass, r, a.K == 0, before, trouble, lane);
}

struct ScoreWs {
    size_t off_ticket, off_rank, zero_bytes;
    RowScratchLayout rs;
};
ScoreWs score_ws_layout(long long rows, int nslices) {
    ScoreWs w;
    size_t o = 0;
    w.off_ticket = o; o += align_up((size_t)rows * 4, 256);
    w.off_rank = o;   o += align_up((size_t)rows * 4, 256);
    w.zero_bytes = o;
    w.rs = row_scratch_layout(o, rows, nslices);
    return w;
}

// Elements of a row that are streamed whatever its start: all of it where every row starts on 16 bytes, else the pieces that lie inside
// it at any start.  Slices are planned for rows that do not start on 16 bytes too, so that the workspace's size does not go by the address.
template <typename DT>
int inner_elems(const void *base, int V, long long stride_b, long long stride_l) {
    constexpr int N = Elem<DT>::N;
    if (base && stream_layout_ok<DT>(base, V, stride_b, stride_l)) return V;
    return V < 2 * N ? 0 : (V - (N - 1)) / N * N;
}
template <typename DT>
SlicePlan score_plan(long long rows, int inner) {
    return plan_slices<DT>(rows, inner, slice_target_ctas());
}

template <typename DT>
int32_t launch_score_cluster(ScoreArgs &a, long long rows, int C, cudaStream_t st) {
    a.nslices = C;
    a.nstages = (a.ntiles_row + C - 1) / C;
    a.own_status = a.L == 1;
    if (!a.own_status) {
        PrepareArgs prep = PrepareArgs();
        prep.zero_b = a.row_status; prep.n_b = a.B;
        DSP_CUDA_TRY(launch_prepare(prep, st));
    }
    static std::atomic<unsigned long long> smem_done{0};
    DSP_CUDA_TRY(allow_shared(score_cluster_kernel<DT>, kClusterTiles * kTileBytes + kFinishArea, smem_done));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(rows * C));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = (size_t)(a.nstages * kTileBytes + kFinishArea);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)C;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = a.own_status ? 1 : 2;
    DSP_CUDA_TRY(cudaLaunchKernelEx(&cfg, score_cluster_kernel<DT>, (const ScoreArgs)a));
    DSP_CUDA_TRY(cudaGetLastError());
    return DSP_OK;
}

template <typename Kernel>
int32_t launch_score_rows(Kernel kernel, long long nblocks, const ScoreArgs &a, cudaStream_t st) {
    DSP_CUDA_TRY(launch_dependent(kernel, (unsigned)nblocks, kThreads, (size_t)a.nstages * kTileBytes, st, a, true));
    DSP_CUDA_TRY(cudaGetLastError());
    return DSP_OK;
}

template <typename DT>
int32_t launch_score(ScoreArgs &a, void *workspace, size_t workspace_bytes, cudaStream_t st) {
    const long long rows = (long long)a.B * a.L;
    a.inner = inner_elems<DT>(a.logits, a.V, a.stride_b, a.stride_l);
    const SlicePlan plan = score_plan<DT>(rows, a.inner);
    a.nslices = plan.nslices;
    a.ntiles_row = (a.inner + tile_elems<DT>() - 1) / tile_elems<DT>();
    const ScoreWs w = score_ws_layout(rows, a.nslices);
    if (workspace_bytes < w.rs.end) return DSP_ERR_WORKSPACE;
    const int C = a.ntiles_row < kMaxCluster ? a.ntiles_row : kMaxCluster;
    // Few rows go to clusters, as long as an SM gets two or three tiles.  Measured (us, cluster / slices and tickets; bf16, 5 alternatives if
    // not said otherwise): 1 row of 152064 8.9 / 13.2, without alternatives 6.4 / 9.6, fp32 9.2 / 15.0; 17 rows 11.6 / 14.3, fp32 15.9 / 14.9;
    // 34 rows 15.5 / 15.3; of 32003 68 rows 11.1 / 12.9, 136 rows 15.6 / 14.2.
    if (C > 1 && a.ntiles_row <= kClusterTiles * kMaxCluster && 2 * rows * a.ntiles_row <= 5 * device_sm_count())
        return launch_score_cluster<DT>(a, rows, C, st);
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    a.rs.row_ticket = reinterpret_cast<unsigned *>(ws + w.off_ticket);
    a.rs.cols = reinterpret_cast<uint2 *>(ws + w.rs.off_cols);
    a.rs.wpart = reinterpret_cast<WarpPartial *>(ws + w.rs.off_wpart);
    a.rank_acc = reinterpret_cast<unsigned *>(ws + w.off_rank);
    const long long nblocks = rows * a.nslices;
    if (nblocks > 0x7FFFFFFFLL) return DSP_ERR_UNSUPPORTED;
    PrepareArgs prep = PrepareArgs();                    // tickets, counts and status words start at zero
    prep.zero_a = reinterpret_cast<uint32_t *>(ws); prep.n_a = (long long)(w.zero_bytes / 4);
    prep.zero_b = a.row_status; prep.n_b = a.B;
    DSP_CUDA_TRY(launch_prepare(prep, st));
    // More than three CTAs an SM: four, with fewer registers and a ring of two tiles, if the finish has room in it.  Measured with three (us,
    // four / three, bf16): 2048 rows of 152064 84.2 / 85.8, 500 with 20 alternatives 46.6 / 53.1; 2000 of 8000 with 5 alternatives 36 / 43; 2048 of
    // 32003 fp32 43.6 / 45.8; five, with one tile: 102.7 for the first and 52.1 for the last.
    if (nblocks > 3ll * device_sm_count() && kFinishBytes + a.nslices * kThreads * 8 <= 2 * kTileBytes) {
        a.nstages = 2;
        static RingSmemDone done;                        // one per kernel
        DSP_CUDA_TRY(allow_ring_smem(score_kernel<DT, 4>, done));
        return launch_score_rows(score_kernel<DT, 4>, nblocks, a, st);
    }
    a.nstages = ring_stages(nblocks);
    static RingSmemDone done;
    DSP_CUDA_TRY(allow_ring_smem(score_kernel<DT, 3>, done));
    return launch_score_rows(score_kernel<DT, 3>, nblocks, a, st);
}

template <typename DT>
size_t score_ws_bytes(int B, int L, int V) {
    const long long rows = (long long)B * L;
    const size_t whole = score_ws_layout(rows, score_plan<DT>(rows, V).nslices).rs.end;
    const size_t part = score_ws_layout(rows, score_plan<DT>(rows, inner_elems<DT>(nullptr, V, 0, 0)).nslices).rs.end;
    return whole > part ? whole : part;
}

int32_t check_score(int32_t B, int32_t L, int32_t V, int32_t dtype) {
    if (B < 0 || L < 1 || V < 1) return DSP_ERR_INVALID_ARG;
    if ((dtype != DSP_F32 && dtype != DSP_BF16) || V > (1 << 30) || (long long)B * L > (1 << 24)) return DSP_ERR_UNSUPPORTED;
    return DSP_OK;
}

}  // namespace
}  // namespace dsp

extern "C" int32_t dsp_token_logprobs_workspace_bytes(int32_t B, int32_t L, int32_t V, int32_t dtype, size_t *bytes) {
    using namespace dsp;
    if (!bytes) return DSP_ERR_INVALID_ARG;
    const int32_t rc = check_score(B, L, V, dtype);
    if (rc != DSP_OK) return rc;
    const int Bq = B > 0 ? B : 1;
    *bytes = dtype == DSP_BF16 ? score_ws_bytes<__nv_bfloat16>(Bq, L, V) : score_ws_bytes<float>(Bq, L, V);
    return DSP_OK;
}

extern "C" int32_t dsp_token_logprobs(const void *logits, int32_t dtype, int32_t B, int32_t L, int32_t V,
                                      int64_t stride_b, int64_t stride_l, const int32_t *row_len,
                                      const int32_t *tokens, int32_t G, float temperature, int32_t K,
                                      float *logp, int32_t *rank, int32_t *top_id, float *top_logit, float *top_logp,
                                      float *lse, float *entropy, uint32_t *row_status,
                                      void *workspace, size_t workspace_bytes, dsp_stream_t stream) {
    using namespace dsp;
    const int32_t rc = check_score(B, L, V, dtype);
    if (rc != DSP_OK) return rc;
    if (G < 0 || K < 0 || !(temperature >= 1e-3f && temperature <= 1e3f)) return DSP_ERR_INVALID_ARG;
    if (K > DSP_MAX_K || G > DSP_MAX_SCORED) return DSP_ERR_UNSUPPORTED;
    if (B == 0) return DSP_OK;
    if (!logits || !lse || !row_status || !workspace) return DSP_ERR_INVALID_ARG;
    if ((G > 0 && (!tokens || !logp)) || (rank && G < 1) || (K > 0 && (!top_id || !top_logit || !top_logp))) return DSP_ERR_INVALID_ARG;
    if (stride_l < V || stride_b < 0 || (B > 1 && stride_b < (int64_t)(L - 1) * stride_l + V)) return DSP_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(workspace) & 255) != 0) return DSP_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(logits) & (dtype == DSP_BF16 ? 1 : 3)) != 0) return DSP_ERR_INVALID_ARG;
    ScoreArgs a = {};
    a.logits = logits;
    a.B = B; a.L = L; a.V = V;
    a.stride_b = stride_b; a.stride_l = stride_l;
    a.row_len = row_len; a.tokens = tokens;
    a.G = G; a.K = K;
    a.inv_t = 1.0 / (double)temperature;
    a.s = (float)(a.inv_t / kLn2);
    a.inv_s = a.inv_t / (double)a.s;
    // What masked logits are raised to: the lowest exponent, by a logit that bf16 holds, for both types.  fl(low s) is the reference of a thread that
    // sees nothing else (with -1e37 its sums were infinite at about every other temperature).
    const float low = kLowest / a.s;
    memcpy(&a.low, &low, 4);
    a.low &= 0xFFFF0000u;
    float held;
    memcpy(&held, &a.low, 4);
    a.low_s = held * a.s;
    if (dtype == DSP_BF16) a.low |= a.low >> 16;
    a.logp = logp; a.rank = rank; a.top_id = top_id; a.top_logit = top_logit; a.top_logp = top_logp;
    a.lse = lse; a.entropy = entropy; a.row_status = row_status;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    return dtype == DSP_BF16 ? launch_score<__nv_bfloat16>(a, workspace, workspace_bytes, st)
                             : launch_score<float>(a, workspace, workspace_bytes, st);
}
