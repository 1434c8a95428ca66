// dsp_distill, dsp_distill_grad: a drafter learns from the teacher's top logits (loss and gradient: dsp.h).
//
// Everything but K values of a row follows from two numbers.  With e_v = 2^(x_v log2e/T - c), c the largest exponent
// among the tokens that the teacher does not name, and S their sum of e_v:
//   q_v = e_v 2^(c - c_all) / S_all,   s = S 2^(c - c_all) / S_all,   dloss/dx_v = e_v * f,
//   f = (2^(c - c_all) / S_all - r / S) / T,
// so the gradient of a row is one exponential and one product per element, with K elements put in afterwards.  S is
// summed over the other tokens alone (the teacher's are taken out of the row before the sum), because s and r / s cannot be had from 1 - sum q
// where the teacher's tokens hold nearly all of the mass.
//
// The floor is one read and one write of the row.  A row is cut into equal slices for a cluster of CTAs, a slice stays in
// its CTA's shared memory between the sums and the gradient (bulk copies in, plain 16-byte stores out), and every warp hands
// four numbers (two references, two sums) to all CTAs of the row over distributed shared memory, once.  The CTAs of an SM belong to
// different rows, so one loads while another sums.
//
// Measured (device time; loss and gradient in one call, K = 32): 2048 rows of 152064 bf16, a tenth of them without weight, 211 us, which is
// 5.6 TB/s or 0.87 of a plain copy's rate; 999 rows of 32003 fp32 49.5 us (0.80), 600 of 152064 148 us (0.77); 512 rows of 152064 bf16 in two calls
// 91 us (0.80; the gradient's call alone 46 us, a copy's rate); 16 rows 7.5 us.  Longer lists cost: 2048 rows, all with weight, K = 32 225 us,
// 64 230, 100 237, 128 239, 256 278.  What bounds the one call is the chain of a row: list, copies, sums, exchange, factors, gradient,
// of which the four or five CTAs of an SM cover most.  On 2048 rows the exchange with a cluster barrier's fences took 250 us, counted stores 228, the loss beside the
// gradient 218 (211 now).  Other forms measured there, before these: clusters that stay and load the next row into a second buffer 434 us, a row in one CTA
// with what does not fit read again from L2 276 us; a cubic for part of the exponentials: within 2%.
#include "stream_core.cuh"

namespace dsp {
namespace {

constexpr int kDT = 256;                        // threads of a CTA: one per teacher slot
static_assert(kDT == DSP_MAX_TEACHER && kDT == kThreads, "one thread per slot");
constexpr int kMaxCluster = 8;
// A CTA's share of a row, 64 KB, unless the cluster is at its largest.  Measured with 40 KB (us, 40 / 64 KB): 1000 rows of 100000 bf16 91 / 75,
// of 110000 96 / 91, of 128256 105 / 100, of 32000 30.0 / 29.5, fp32 999 of 32003 52.4 / 48.9, 1000 of 64000 93 / 88, 600 of 152064 148 / 148; with
// 80 KB 2048 rows of 152064 bf16 took 261 instead of 225, the others the same.
constexpr int kSliceVecs = 4096;
constexpr uint32_t kNoEntry = 0xFFFFFFFFu;      // state: a slot that takes no part

struct DistillArgs {
    const void *x;
    long long sb, sl;
    int L, V, K, C, log2_c;                     // C: CTAs of a row
    int buf_vecs;                               // 16-byte vectors that a CTA's buffer holds
    const int32_t *id, *count;
    const float *val, *tlse, *weight;
    double inv_t, inv_s;                        // 1 / T, and back from exponents: 1 / (s T)
    float s;                                    // log2(e) / T in 32 bits: all exponents of a row are multiples of it
    float *loss, *accept, *lse, *state;
    void *g;
    long long gsb, gsl;
    uint32_t *status;
};

// What a warp knows of its share of the row, handed to all CTAs of the row.
struct Part {
    float c, S;              // the other tokens: reference, sum against it
    float ct, E;             // the teacher's tokens that the warp's slots name in this slice: the same
};
struct CopyBar {
    uint64_t bar;
    int timed_out;
};
struct Place {               // of a CTA's slice: worked out by one thread
    const void *x;
    void *g;
    int h, n, lo, hi, p0, p1;
    float w;
};
struct Known {               // of the row, after the exchange
    float cs, S, c_all, to_all, all;
    float f, c_f;            // gradient of the others: f 2^(x s - c_f)
    double r;
    int none;
};
struct Shared : CopyBar {
    uint64_t got;                               // clusters: what the row's CTAs send has arrived
    Known known;
    Place place;
    __align__(16) Part part[kMaxCluster * kWarps];
    float xk[kDT];                              // first CTA: the teacher's tokens under the student
    __align__(16) int id[kDT];
    double red[kWarps][3];
};

// Stores into another CTA of the cluster that are counted, in bytes, by a barrier there: no fence is needed on either side.  For launches with
// clusters alone.
__device__ __forceinline__ void send_counted(uint32_t addr, uint32_t bar, float v0, float v1, float v2, float v3) {
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];"
                 ::"r"(addr), "f"(v0), "f"(v1), "f"(v2), "f"(v3), "r"(bar) : "memory");
}
__device__ __forceinline__ void send_counted(uint32_t addr, uint32_t bar, float v) {
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.f32 [%0], %1, [%2];" ::"r"(addr), "f"(v), "r"(bar) : "memory");
}
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// A row in 16-byte pieces: piece i holds the elements [i N - h, (i + 1) N - h), h the row's distance from the boundary before it.
// Pieces lo .. hi-1 lie inside the row; of the first and the last a part may lie outside, which is neither read nor written.
template <typename DT>
struct Pieces {
    static constexpr int N = Elem<DT>::N;
    int h, n, lo, hi;
    Pieces() = default;
    __device__ __forceinline__ Pieces(const DT *row, int V) {
        h = (int)((reinterpret_cast<uintptr_t>(row) / sizeof(DT)) % N);
        n = (h + V + N - 1) / N;
        lo = h ? 1 : 0;
        hi = (h + V) / N;
    }
};
// Calls at(element, place) for the elements of the partly outside pieces among [a, b), one element a thread; outside: element -1.
template <typename DT, typename At>
__device__ __forceinline__ void edges(const Pieces<DT> &p, int V, int a, int b, int tid, At at) {
    constexpr int N = Elem<DT>::N;
    auto one = [&](int piece, int e) {
        const int v = piece * N + e - p.h;
        at(v >= 0 && v < V ? v : -1, (piece - a) * N + e);
    };
    if (p.lo == 1 && a == 0 && tid < N) one(0, tid);
    if (p.hi < p.n && p.n - 1 >= p.lo && p.n == b && tid >= 32 && tid < 32 + N) one(p.n - 1, tid - 32);
}

// Pieces [a, b) of the row into the buffer: one thread sends the copies of whole pieces, the elements of the others are read one a thread
// (outside of the row: -inf).  A barrier of the CTA lies between the last use of the buffer (fenced) and the copies; complete after
// take_copies and a barrier of the CTA.
template <typename DT>
__device__ __forceinline__ void send_copies(const DT *row, const Pieces<DT> &p, int a, int b, DT *buf, CopyBar &sh) {
    constexpr int N = Elem<DT>::N;
    const int l = max(a, p.lo), u = min(b, p.hi);
    const uint32_t bytes = u > l ? (uint32_t)(u - l) * 16u : 0u;
    mbar_expect_tx(&sh.bar, bytes);
    const char *src = reinterpret_cast<const char *>(row + ((long long)l * N - p.h));
    char *dst = reinterpret_cast<char *>(buf + (size_t)(l - a) * N);
    constexpr uint32_t kPiece = 16384;
    for (uint32_t o = 0; o < bytes; o += kPiece) bulk_load(dst + o, src + o, min(kPiece, bytes - o), &sh.bar);
}
template <typename DT>
__device__ __forceinline__ void read_edges(const DT *row, const Pieces<DT> &p, int V, int a, int b, DT *buf) {
    if (p.lo == 0 && p.hi == p.n) return;
    edges<DT>(p, V, a, b, threadIdx.x, [&](int v, int place) {
        if (v >= 0) buf[place] = row[v];
        else if constexpr (Elem<DT>::N == 8) reinterpret_cast<unsigned short *>(buf)[place] = 0xFF80u;
        else reinterpret_cast<uint32_t *>(buf)[place] = 0xFF800000u;
    });
}

// Waits for a buffer's copies (or what `bar` counts), asleep for a microsecond at a time: other CTAs of the SM have the issue slots meanwhile.
__device__ __forceinline__ void take(uint64_t &bar, CopyBar &sh, uint32_t parity, int turns = 2) {
    const long long t0 = clock64();
    for (int turn = 0; turn < turns; ++turn) {
        do {
            uint32_t ok;
            asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\nselp.u32 %0, 1, 0, p;\n}"
                         : "=r"(ok) : "r"(smem_addr(&bar)), "r"(parity), "r"(1000u) : "memory");
            if (ok) return;
        } while (clock64() - t0 < (turn + 1) * kWaitCycles);
        sh.timed_out = 1;                       // once more, so that no copy is under way into a buffer that is used again
    }
}

__device__ __forceinline__ void take_copies(CopyBar &sh, uint32_t parity) { take(sh.bar, sh, parity); }

template <typename DT> __device__ __forceinline__ float elem_of(const DT *buf, int i) { return Elem<DT>::load1(buf + i); }
template <typename DT> __device__ __forceinline__ void hide(DT *buf, int i) {
    if constexpr (sizeof(DT) == 2) reinterpret_cast<unsigned short *>(buf)[i] = 0xFF80u;
    else reinterpret_cast<uint32_t *>(buf)[i] = 0xFF800000u;
}
template <typename DT> __device__ __forceinline__ DT rounded(float v) {
    if constexpr (sizeof(DT) == 2) return __float2bfloat16(v);
    else return v;
}

// Largest of a warp (NaN aside) and sum over it.
__device__ __forceinline__ float max_of_warp(float v) {
    float m;
    asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(m) : "f"(v));
    return m;
}
__device__ __forceinline__ float sum_of_warp(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

// Sum of 2^(x s - c) over the buffer's pieces, by this thread's share.  The reference c of a warp is the largest exponent of its
// first pieces: an fp32 sum also holds what exceeds it, so the others need no look at their maximum.  Where a sum passes 2^64 (or a
// logit is not finite) the warp sums once more against its true maximum, so that no sum is lost below another warp's reference.
// Two logits an instruction where the hardware has one (2048 rows of 152064 bf16: 256 to 252 us at the time).
template <typename DT>
__device__ __forceinline__ void add_piece(const uint4 &v, float s, float c, unsigned long long &S) {
    const unsigned long long s2 = pack2(s, s), nc2 = pack2(-c, -c);
#pragma unroll
    for (int e = 0; e < Elem<DT>::N; e += 2) {
        float a0, a1;
        unpack2(fma2(pack2(Elem<DT>::get(v, e), Elem<DT>::get(v, e + 1)), s2, nc2), a0, a1);
        S = add2(S, pack2(ex2_approx(a0), ex2_approx(a1)));
    }
}
__device__ __forceinline__ float both(unsigned long long S) {
    float a, b;
    unpack2(S, a, b);
    return a + b;
}
template <typename DT>
__device__ __forceinline__ void sum_pieces(const uint4 *buf, int n, float s, float &c, float &S) {
    const int tid = threadIdx.x, full = n / kDT, rest = n % kDT;       // whole rounds of the CTA, pieces of the last one
    const uint4 *at = buf + tid;
    float m = -CUDART_INF_F;
    if (tid < n) m = Elem<DT>::vmax(at[0]);
    if (tid + kDT < n) m = fmaxf(m, Elem<DT>::vmax(at[kDT]));
    float c1 = fmaxf(max_of_warp(m) * s, kLowest);
    unsigned long long s0 = 0ull, t0 = 0ull;             // pairs of sums
    int k = full;
    for (; k >= 2; k -= 2, at += 2 * kDT) {
        const uint4 v = at[0], w = at[kDT];
        add_piece<DT>(v, s, c1, s0);
        add_piece<DT>(w, s, c1, t0);
    }
    if (k) { add_piece<DT>(at[0], s, c1, s0); at += kDT; }
    if (tid < rest) add_piece<DT>(at[0], s, c1, t0);
    float sum = both(add2(s0, t0));
    if (__any_sync(0xFFFFFFFFu, !(sum < 0x1p64f))) {
        for (int i = tid; i < n; i += kDT) m = fmaxf(m, Elem<DT>::vmax(buf[i]));
        c1 = fmaxf(max_of_warp(m) * s, kLowest);
        s0 = 0ull;
        for (int i = tid; i < n; i += kDT) add_piece<DT>(buf[i], s, c1, s0);
        sum = both(s0);
    }
    // with what the chunks before gave
    const float cn = fmaxf(c, c1);
    S = (S != 0.f ? S * ex2_approx(c - cn) : 0.f) + (sum != 0.f ? sum * ex2_approx(c1 - cn) : 0.f);
    c = cn;
}

// f * 2^(x s - c) of a piece, rounded once.
template <typename DT>
__device__ __forceinline__ uint4 turned(const uint4 &v, float s, float c, float f) {
    constexpr int N = Elem<DT>::N;
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < N; e += 2) {
        float a0, a1;
        unpack2(fma2(pack2(Elem<DT>::get(v, e), Elem<DT>::get(v, e + 1)), pack2(s, s), pack2(-c, -c)), a0, a1);
        unpack2(mul2(pack2(ex2_approx(a0), ex2_approx(a1)), pack2(f, f)), a0, a1);
        if constexpr (N == 8) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(a0, a1);
            w[e / 2] = *reinterpret_cast<const uint32_t *>(&b);
        } else {
            w[e] = __float_as_uint(a0);
            w[e + 1] = __float_as_uint(a1);
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Element e of a piece, to memory.
template <typename DT>
__device__ __forceinline__ void put_one(DT *to, const uint4 &t, int e) {
    if constexpr (Elem<DT>::N == 8) {
        const uint32_t w = e < 2 ? t.x : e < 4 ? t.y : e < 6 ? t.z : t.w;
        *reinterpret_cast<unsigned short *>(to) = (unsigned short)(e & 1 ? w >> 16 : w);
    } else {
        *to = Elem<DT>::get(t, e);
    }
}
// The gradient of pieces [a, b) from their logits in the buffer, the teacher's tokens aside.  Rows of the gradient that start where the
// logits' do within 16 bytes take whole pieces (then the first `skip` threads may stay away), others are written element by element.
template <typename DT>
__device__ __forceinline__ bool same_start(const DT *grow, const Pieces<DT> &p) {
    return (int)((reinterpret_cast<uintptr_t>(grow) / sizeof(DT)) % Elem<DT>::N) == p.h;
}
template <typename DT>
__device__ __forceinline__ void write_pieces(DT *grow, const Pieces<DT> &p, int V, int a, int b, DT *buf, float s, float c, float f, int skip = 0) {
    constexpr int N = Elem<DT>::N;
    uint4 *bp = reinterpret_cast<uint4 *>(buf);
    if (same_start(grow, p)) {
        const int l = max(a, p.lo), u = min(b, p.hi);
        uint4 *gp = reinterpret_cast<uint4 *>(grow + ((long long)l * N - p.h));
        const uint4 *from = bp + (l - a);
        const int me = (int)threadIdx.x - skip, step = kDT - skip;
        int i = me;
        for (; i + step < u - l; i += 2 * step) {
            const uint4 v0 = from[i], v1 = from[i + step];
            gp[i] = turned<DT>(v0, s, c, f);
            gp[i + step] = turned<DT>(v1, s, c, f);
        }
        if (i < u - l) gp[i] = turned<DT>(from[i], s, c, f);
        if (p.lo == 0 && p.hi == p.n) return;
        edges<DT>(p, V, a, b, me, [&](int v, int place) {
            if (v < 0) return;
            put_one<DT>(grow + v, turned<DT>(bp[place / N], s, c, f), place % N);
        });
    } else {
        for (int i = threadIdx.x; i < b - a; i += kDT) bp[i] = turned<DT>(bp[i], s, c, f);
        __syncthreads();
        const int v0 = max(0, a * N - p.h), v1 = min(V, b * N - p.h);
        for (int v = v0 + threadIdx.x; v < v1; v += kDT) grow[v] = buf[v + p.h - a * N];
    }
}

// Zeros as the gradient of the elements [v0, v1).
template <typename DT>
__device__ void store_zeros(DT *grow, int v0, int v1) {
    constexpr int N = Elem<DT>::N;
    const int h = (int)((reinterpret_cast<uintptr_t>(grow) / sizeof(DT)) % N);
    const int first = min(v1, (v0 + h + N - 1) / N * N - h), last = max(first, (v1 + h) / N * N - h);
    for (int v = v0 + threadIdx.x; v < first; v += kDT) grow[v] = rounded<DT>(0.f);
    for (int v = last + threadIdx.x; v < v1; v += kDT) grow[v] = rounded<DT>(0.f);
    uint4 *g4 = reinterpret_cast<uint4 *>(grow + first);
    for (int i = threadIdx.x; i < (last - first) / N; i += kDT) g4[i] = make_uint4(0u, 0u, 0u, 0u);
}

// The list of a row, one slot a thread (ids: all slots', complete): of equal ids the first slot counts; its probability.  The sum of all: P, or
// with the teacher's log-sum-exp of each warp in red[warp][0].  Every thread of the CTA.
__device__ __forceinline__ void probabilities(const DistillArgs &a, int &id, float t, float t_lse, const int *ids, double (*red)[3], double &lp,
                                              double &pk, double &P) {
    const int tid = threadIdx.x, lane = tid & 31, warp = warp_index();
    if (id >= 0) {                              // of equal ids the first slot counts
        bool twice = false;
        const int4 *quads = reinterpret_cast<const int4 *>(ids);
        for (int j = 0; j < tid >> 2; ++j) {
            const int4 o = quads[j];
            twice |= o.x == id || o.y == id || o.z == id || o.w == id;
        }
        for (int j = tid & ~3; j < tid; ++j) twice |= ids[j] == id;
        if (twice) id = -1;
    }
    lp = -CUDART_INF;
    pk = P = 0.0;
    if (a.tlse) {
        if (id >= 0) lp = (double)t * a.inv_t - (double)t_lse;
        if (id >= 0) pk = exp(lp);
        if (warp * 32 < a.K) {
            const double Pw = warp_sum(pk);
            if (lane == 0) red[warp][0] = Pw;
        }
    } else {                                    // softmax over the K tokens
        const float m0 = warp_max(id >= 0 ? t : -CUDART_INF_F);
        const bool nan0 = __any_sync(0xFFFFFFFFu, id >= 0 && t != t);
        if (lane == 0) red[warp][0] = nan0 ? CUDART_NAN : (double)m0;
        __syncthreads();
        double m = red[0][0];
        for (int i = 1; i * 32 < a.K; ++i) {
            const double o = red[i][0];
            if (m == m && !(o <= m)) m = o;     // a NaN stays
        }
        const double e = id >= 0 && m != -CUDART_INF ? exp(((double)t - m) * a.inv_t) : 0.0;
        const double z0 = warp * 32 < a.K ? warp_sum(m != m ? m : e) : 0.0;
        if (lane == 0) red[warp][1] = z0;
        __syncthreads();
        double z = 0.0;
        for (int i = 0; i * 32 < a.K; ++i) z += red[i][1];
        P = z == 0.0 ? 0.0 : z / z;             // 1, or NaN
        if (id >= 0 && z != 0.0) {
            pk = e / z;
            lp = ((double)t - m) * a.inv_t - log(z);
        }
    }
}

// Loss and what else a row is told, by the first n threads of a CTA, all that have slots among them; x: the slot's token under the student.  The student's mass of the teacher's
// tokens is summed once more in 64 bits: with dloss = (s - r) dS / S + (1 - s) dE / E, an error of the other tokens' sum S nearly cancels where
// the drafter is near the teacher, one of E does not (mean error of losses around 0.03: 1e-6 of themselves with 32 bits).
__device__ __forceinline__ void tell_row(const DistillArgs &a, unsigned row, int id, double lp, double pk, double P, float xt, const Known &kn,
                                         double (*red)[3], int n) {
    const int tid = threadIdx.x, lane = tid & 31, warp = warp_index();
    float *state = a.state ? a.state + (long long)row * (a.K + 4) : nullptr;
    if (warp * 32 < a.K) {
        double h = 0.0, m = 0.0, e = 0.0;
        if (id >= 0) {
            if (pk != 0.0) h = pk * (lp - (double)xt * a.inv_t);
            e = exp((double)xt * a.inv_t - (double)kn.c_all * a.inv_s);
            m = fmin(pk, e / (double)kn.all);
        }
        h = warp_sum(h);
        m = warp_sum(m);
        e = warp_sum(e);
        if (lane == 0) { red[warp][0] = h; red[warp][1] = m; red[warp][2] = e; }
    }
    if (state && tid < a.K && id < 0) reinterpret_cast<uint32_t *>(state)[4 + tid] = kNoEntry;
    asm volatile("bar.sync 1, %0;" ::"r"(n) : "memory");
    if (tid == 0) {
        double H = 0.0, accept = 0.0, E = 0.0;
        for (int i = 0; i * 32 < a.K; ++i) { H += red[i][0]; accept += red[i][1]; E += red[i][2]; }
        const bool ok = kn.all > 0.f && kn.all < CUDART_INF_F && kn.c_all > kLowest && kn.c_all < CUDART_INF_F;
        const float cs = kn.cs, S = kn.S;
        const double others = S != 0.f ? (double)S * exp(((double)cs - (double)kn.c_all) * a.inv_s) : 0.0, total = others + E;
        const double lse = ok ? (double)kn.c_all * a.inv_s + kLn2 * log2(total) : CUDART_NAN;
        const double r = kn.r;
        double loss = kn.none ? 0.0 : H + P * lse;
        if (r != 0.0) loss += r * (log(r) - ((double)cs * a.inv_s + kLn2 * log2((double)S) - lse));
        const double s = others / total;
        a.loss[row] = ok ? (float)loss : CUDART_NAN_F;
        if (a.lse) a.lse[row] = (float)lse;
        if (a.accept) a.accept[row] = (float)(accept + (r < s ? r : s));
        if (state) { state[0] = kn.c_f; state[1] = kn.f; state[2] = 0.f; state[3] = 0.f; }
        if (a.status && (!ok || !(P < CUDART_INF) || (a.tlse && !(a.tlse[row] < CUDART_INF_F)))) atomicOr(&a.status[row / (unsigned)a.L], DSP_ROW_NONFINITE_INPUT);
    }
}
// A row that is not read.
__device__ __forceinline__ void tell_nothing(const DistillArgs &a, unsigned row) {
    const int tid = threadIdx.x;
    float *state = a.state ? a.state + (long long)row * (a.K + 4) : nullptr;
    if (tid == 0) {
        a.loss[row] = 0.f;
        if (a.accept) a.accept[row] = 0.f;
        if (a.lse) a.lse[row] = -CUDART_INF_F;
        if (state) { state[0] = -kRefFloor; state[1] = 0.f; state[2] = 0.f; state[3] = 0.f; }
    }
    if (state && tid < a.K) reinterpret_cast<uint32_t *>(state)[4 + tid] = kNoEntry;
}
__device__ __forceinline__ float lost_if(int timed_out) { return timed_out ? CUDART_NAN_F : 0.f; }
// What follows from the sums of a row's n parts, by one warp (P: the list's sum, t_lse: the teacher's log-sum-exp; lost: 0, or NaN where copies
// or parts did not all come in time: then everything that follows from the sums is NaN).
//
// r = 1 - P has the rounding of the teacher's log-sum-exp in it, 2^-24 |t_lse| and as much again for whoever summed it, and a few 2^-24 of the
// sum's own: where the list is all that the teacher allows, that is all that r is.  r log s would turn it into a loss of any size where the
// drafter gives the others next to nothing (a common mask: s = 0, or e^-10000), so there it counts as nothing.  Where s is above r / 1024 the
// formula stays: its term is within 7 r then.
//
// All of this is in 32 bits, because the gradient waits for it (with it, five CTAs an SM and the loss out of the way 2048 rows of 152064 went from 480 us
// to 368): the sums are off by
// a few 2^-24, the two quotients of f and the q of a listed token by 2^-22.  f and q - p are differences, so the gradient's error is some
// 2^-21 of q_v, not of itself: 2^-21 / (1 - r/s) of itself for the others, 5e-5 where r/s is within a hundredth of 1.
__device__ __forceinline__ Known known_of(const DistillArgs &a, const Part *parts, int n, double P, float t_lse, float lost, int lane) {
    Part q[kMaxCluster * kWarps / 32];
    float cs = kLowest, cl = kLowest, S = lost, E = 0.f;
#pragma unroll
    for (int i = 0; i < kMaxCluster * kWarps / 32; ++i) {
        q[i] = lane + 32 * i < n ? parts[lane + 32 * i] : Part{kLowest, 0.f, kLowest, 0.f};
        cs = fmaxf(cs, q[i].c);
        cl = fmaxf(cl, q[i].ct);
    }
    cs = max_of_warp(cs);
    cl = max_of_warp(cl);
#pragma unroll
    for (int i = 0; i < kMaxCluster * kWarps / 32; ++i) {
        const float w2 = ex2_approx(q[i].c - cs);
        // far below the reference: nothing, but NaN and infinite sums stay visible
        S += w2 == 0.f && q[i].S < CUDART_INF_F ? 0.f : q[i].S * w2;
        E += q[i].E != 0.f ? q[i].E * ex2_approx(q[i].ct - cl) : 0.f;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        S += __shfl_xor_sync(0xFFFFFFFFu, S, o);
        E += __shfl_xor_sync(0xFFFFFFFFu, E, o);
    }
    Known kn;
    kn.cs = cs;
    kn.S = S;
    kn.c_all = fmaxf(cs, cl);
    kn.to_all = ex2_approx(cs - kn.c_all);
    kn.all = (S != 0.f ? S * kn.to_all : 0.f) + (E != 0.f ? E * ex2_approx(cl - kn.c_all) : 0.f);
    const double r = a.tlse ? 1.0 - P : 0.0;
    kn.r = r < 0.0 ? 0.0 : r;               // NaN stays
    const float rest = (float)kn.r;
    if (rest > 0.f && rest <= 0x1p-23f * (fabsf(t_lse) + 4.f) && S * kn.to_all < rest * 0x1p-10f * kn.all) kn.r = 0.0;
    kn.none = !a.tlse && P == 0.0;           // the list says nothing: no gradient
    kn.f = kn.none || S == 0.f ? 0.f : (__fdividef(kn.to_all, kn.all) - __fdividef((float)kn.r, S)) * (float)a.inv_t;
    kn.c_f = S != 0.f ? cs : -kRefFloor;    // nothing to scale: every exponential is 0
    return kn;
}

// CTAS: of an SM.
template <typename DT, bool GRAD, int CTAS>
__global__ void __launch_bounds__(kDT, CTAS) distill_kernel(const DistillArgs a) {
    constexpr int N = Elem<DT>::N;
    extern __shared__ __align__(128) unsigned char ring[];
    __shared__ Shared sh;
    DT *buf = reinterpret_cast<DT *>(ring);
    const int tid = threadIdx.x, lane = tid & 31, warp = warp_index();
    const int C = a.C, rank = C > 1 ? (int)cluster_rank() : 0;
    const unsigned row32 = blockIdx.x >> a.log2_c;
    const long long row = row32;
    // ---- the teacher's list, one slot a thread: its probabilities are formed while the copies are under way ----
    int id = -1;
    float t = -CUDART_INF_F;
    const bool tail = a.tlse != nullptr;
    const float t_lse = tail ? a.tlse[row] : 0.f;
    if (tid < a.K) {
        id = a.id[row * a.K + tid];
        t = a.val[row * a.K + tid];
        const int n = a.count ? a.count[row] : a.K;
        if (tid >= n || id < 0 || id >= a.V) id = -1;
    }
    if (tid == kDT - 1) {                       // the warp that has a list only if it is a long one
        Place &at = sh.place;
        const float w0 = a.weight ? a.weight[row] : 1.f;
        const unsigned b0 = row32 / (unsigned)a.L, l0 = row32 - b0 * (unsigned)a.L;
        const DT *x0 = reinterpret_cast<const DT *>(a.x) + b0 * a.sb + l0 * a.sl;
        const Pieces<DT> p(x0, a.V);
        at.x = x0;
        if (GRAD) at.g = reinterpret_cast<DT *>(a.g) + b0 * a.gsb + l0 * a.gsl;
        at.h = p.h; at.n = p.n; at.lo = p.lo; at.hi = p.hi;
        at.p0 = (int)(((unsigned)p.n * (unsigned)rank) >> a.log2_c);
        at.p1 = (int)(((unsigned)p.n * (unsigned)(rank + 1)) >> a.log2_c);
        at.w = w0;
        sh.timed_out = 0;
        mbar_init(&sh.bar, 1);
        mbar_init(&sh.got, 1);
        mbar_init_fence();
        if (w0 != 0.f) send_copies<DT>(x0, p, at.p0, min(at.p1, at.p0 + a.buf_vecs), buf, sh);
    }
    sh.id[tid] = id;
    __syncthreads();
    const DT *x = reinterpret_cast<const DT *>(sh.place.x);
    DT *g = reinterpret_cast<DT *>(sh.place.g);
    Pieces<DT> p;
    p.h = sh.place.h; p.n = sh.place.n; p.lo = sh.place.lo; p.hi = sh.place.hi;
    const int p0 = sh.place.p0, p1 = sh.place.p1;
    const float w = sh.place.w;
    float *state = a.state ? a.state + row * (a.K + 4) : nullptr;
    if (w == 0.f) {                             // the whole cluster alike
        if (GRAD) store_zeros<DT>(g, max(0, p0 * N - p.h), min(a.V, p1 * N - p.h));
        if (rank == 0) tell_nothing(a, row32);
        return;
    }
    if (C > 1) cluster_arrive_empty();
    const int chunks = p1 - p0 <= a.buf_vecs ? 1 : (p1 - p0 + a.buf_vecs - 1) / a.buf_vecs;
    int q0 = p0, q1 = min(p1, p0 + a.buf_vecs);
    uint32_t parity = 0;
    read_edges<DT>(x, p, a.V, q0, q1, buf);
    auto send = [&]() {
        if (tid == 0) send_copies<DT>(x, p, q0, q1, buf, sh);
        read_edges<DT>(x, p, a.V, q0, q1, buf);
    };
    double lp, pk, P;                           // log p_k, p_k, their sum (tail: of the warp's, in sh.red)
    probabilities(a, id, t, t_lse, sh.id, sh.red, lp, pk, P);
    if (C > 1) {
        const int known = __syncthreads_count(id >= 0);
        if (tid == 0) mbar_expect_tx(&sh.got, (uint32_t)(C * kWarps * sizeof(Part)) + (rank == 0 ? 4u * (uint32_t)known : 0u));
        cluster_wait();                         // the other CTAs are there
    }
    const int piece = id >= 0 ? (p.h + id) / N : -1;      // where the slot's token lies
    const bool mine = piece >= p0 && piece < p1;

    // ---- the slice: the teacher's tokens taken out, the others summed ----
    float xk = 0.f, c = kLowest, Sc = 0.f;
    for (int k = 0;;) {
        if (warp == 0) take_copies(sh, parity);
        parity ^= 1u;
        __syncthreads();                        // the edges are in place too
        if (sh.timed_out) Sc = CUDART_NAN_F;    // a copy that came too late: no sum, for all of the row's CTAs
        if (piece >= q0 && piece < q1) {
            const int at = p.h + id - q0 * N;
            xk = elem_of<DT>(buf, at);
            hide<DT>(buf, at);
        }
        __syncthreads();
        sum_pieces<DT>(reinterpret_cast<const uint4 *>(buf), q1 - q0, a.s, c, Sc);
        if (++k >= chunks) break;
        fence_async();
        __syncthreads();
        q0 = q1;
        q1 = min(p1, q1 + a.buf_vecs);
        send();
    }

    // ---- what the warp knows, to every CTA of the row: all that the gradient waits for is in single precision ----
    const double zs = (double)xk * (double)a.s; // the token's exponent
    Part w1 = {c, sum_of_warp(Sc), kLowest, 0.f};
    if (warp * 32 < a.K) {                      // the warps that have slots
        w1.ct = max_of_warp(mine && (float)zs > kLowest ? (float)zs : kLowest);
        w1.E = sum_of_warp(mine ? ex2_approx((float)(zs - (double)w1.ct)) : 0.f);
    }
    if (C > 1) {
        if (mine) send_counted(at_rank(&sh.xk[tid], 0), at_rank(&sh.got, 0), xk);
        if (lane < C) send_counted(at_rank(&sh.part[rank * kWarps + warp], lane), at_rank(&sh.got, lane), w1.c, w1.S, w1.ct, w1.E);
        if (warp == 0) take(sh.got, sh, 0u, 4); // longer than a CTA waits for its copies: what it sends arrives before this one leaves
    } else {
        if (mine) sh.xk[tid] = xk;
        if (lane == 0) sh.part[warp] = w1;
        __syncthreads();
    }

    // ---- the row, by one warp for all ----
    if (warp == 0) {
        if (tail)
            for (int i = 0; i * 32 < a.K; ++i) P += sh.red[i][0];
        const Known kn = known_of(a, sh.part, C * kWarps, P, t_lse, lost_if(*static_cast<volatile int *>(&sh.timed_out)), lane);
        if (lane == 0) sh.known = kn;
    }
    __syncthreads();
    const float c_all = sh.known.c_all, all = sh.known.all, f = sh.known.f, c_f = sh.known.c_f;
    const bool none = sh.known.none;
    float gk = 0.f;                             // the slot's gradient for a weight of 1
    if (mine) gk = none ? 0.f : (float)(((double)__fdividef(ex2_approx((float)(zs - (double)c_all)), all) - pk) * a.inv_t);
    if (state && mine) state[4 + tid] = gk;
    // Loss and what else the row is told, by the first CTA: while the others write the gradient by the warps with slots alone, if those are few and
    // the pieces are whole ones (us, so / by all warps before the gradient: 2048 rows of 152064 bf16 225 / 258; K = 64: 230 / 261, 1000 of 32000
    // 30.1 / 31.1, 999 of 32003 fp32 48.6 / 51.4).  Lists of 65 to 128 would gain as well (K = 100: 230 / 237, 31.2 / 32.2, 50.7 / 53.5).
    int skip = 0;
    if (rank == 0) {
        const int listed = (a.K + 31) / 32 * 32;
        if (GRAD && listed <= kDT / 4 && chunks == 1 && same_start(g, p)) skip = listed;
        if (skip == 0 || tid < skip)
            tell_row(a, row32, id, lp, pk, P, tid < a.K && id >= 0 ? sh.xk[tid] : 0.f, sh.known, sh.red, skip ? skip : kDT);
    }
    if constexpr (GRAD) {
        for (int k = 0;;) {
            // one chunk: it is in the buffer still, without the teacher's tokens; several: once more from the first on
            if (chunks > 1) {
                q0 = p0 + k * a.buf_vecs;
                q1 = min(p1, q0 + a.buf_vecs);
                fence_async();
                __syncthreads();
                send();
                if (warp == 0) take_copies(sh, parity);
                parity ^= 1u;
                __syncthreads();
            }
            if (tid >= skip) write_pieces<DT>(g, p, a.V, q0, q1, buf, a.s, c_f, chunks > 1 && sh.timed_out ? CUDART_NAN_F : f * w, skip);
            __syncthreads();                    // the token's own element comes after the piece that it lies in
            if (piece >= q0 && piece < q1) g[id] = rounded<DT>(gk * w);
            if (++k >= chunks) break;
        }
    }
    if (tid == 0 && sh.timed_out && a.status) atomicOr(&a.status[row32 / (unsigned)a.L], DSP_ROW_TIMEOUT);
}

// ---- the loss alone, of many rows: nothing has to stay, so a CTA streams a row of its own (stream_core.cuh) ----

// Takes element e out of a piece and returns it.
template <typename DT>
__device__ __forceinline__ float take_out(uint4 &v, int e) {
    float x = 0.f;
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < Elem<DT>::N; ++i) {
        if (i != e) continue;
        x = Elem<DT>::get(v, i);
        if constexpr (Elem<DT>::N == 8) w[i >> 1] = (i & 1) ? (w[i >> 1] & 0x0000FFFFu) | 0xFF800000u : (w[i >> 1] & 0xFFFF0000u) | 0xFF80u;
        else w[i] = 0xFF800000u;
    }
    v = make_uint4(w[0], w[1], w[2], w[3]);
    return x;
}

// As add_piece, without the register pairs, which cost this kernel spills (512 rows of 152064 in two calls 91 us, with them 93).
template <typename DT>
__device__ __forceinline__ void add_single(const uint4 &v, float s, float c, float &S0, float &S1) {
#pragma unroll
    for (int e = 0; e < Elem<DT>::N; e += 2) {
        S0 += ex2_approx(fmaf(Elem<DT>::get(v, e), s, -c));
        S1 += ex2_approx(fmaf(Elem<DT>::get(v, e + 1), s, -c));
    }
}

// The sums of a row without the teacher's tokens.  These are sorted by place; every warp walks through them with the tiles, and the thread
// that has a token takes it out and notes it.
template <typename DT, typename List>
struct LossPass {
    static constexpr bool kOwnTile = true;
    List &make_list;          // forms the list while the first tiles are under way
    const int *place;         // elements of the streamed part, ascending, then one behind all
    float *xk;
    float s;
    int token = 0, next = 0;
    float c = kLowest, S = 0.f, ct = kLowest, E = 0.f;
    bool first = true;

    __device__ __forceinline__ LossPass(List &list, const int *pl, float *x, float scale) : make_list(list), place(pl), xk(x), s(scale) {}
    __device__ __forceinline__ void begin() {
        make_list();
        next = place[0];
    }
    __device__ __forceinline__ void hand_in() {}
    __device__ __forceinline__ void add_token(float x) {
        const float c1 = fmaxf(ct, x * s);
        E = (E != 0.f ? E * ex2_approx(ct - c1) : 0.f) + ex2_approx((float)((double)x * (double)s - (double)c1));
        ct = c1;
    }
    template <bool RAGGED>
    __device__ __forceinline__ float tile(const uint4 (&t)[kVpt], int, int tid, int base, float &, unsigned long long &, unsigned long long &) {
        constexpr int N = Elem<DT>::N;
        uint4 v[kVpt];
#pragma unroll
        for (int j = 0; j < kVpt; ++j) v[j] = t[j];
        for (; next < base + tile_elems<DT>(); next = place[++token]) {
            const int q = (next - base) / N;                     // the token's piece of the tile
            if (q % kThreads != tid) continue;
            float x = 0.f;
#pragma unroll
            for (int j = 0; j < kVpt; ++j)
                if (q / kThreads == j) x = take_out<DT>(v[j], next % N);
            xk[token] = x;
            add_token(x);
        }
        if (first) {
            first = false;
            c = fmaxf(max_of_warp(fmaxf(Elem<DT>::vmax(v[0]), Elem<DT>::vmax(v[1]))) * s, kLowest);
        }
        float s0 = S, s1 = 0.f;
#pragma unroll
        for (int j = 0; j < kVpt; ++j) add_single<DT>(v[j], s, c, s0, s1);
        if (__any_sync(0xFFFFFFFFu, !(s0 + s1 < 0x1p64f))) {     // against a new reference, as in sum_pieces
            float m = Elem<DT>::vmax(v[0]);
#pragma unroll
            for (int j = 1; j < kVpt; ++j) m = fmaxf(m, Elem<DT>::vmax(v[j]));
            const float c1 = fmaxf(max_of_warp(m) * s, c);
            s0 = S != 0.f ? S * ex2_approx(c - c1) : 0.f;
            s1 = 0.f;
#pragma unroll
            for (int j = 0; j < kVpt; ++j) add_single<DT>(v[j], s, c1, s0, s1);
            c = c1;
        }
        S = s0 + s1;
        return 0.f;
    }
};

// Shared memory behind the ring: ids, places, logits of the list.
__host__ __device__ inline int loss_list_words(int K) { return (K + 3) / 4 * 4 + (K + 4) / 4 * 4 + K; }

template <typename DT>
__global__ void __launch_bounds__(kThreads, 3) distill_loss_kernel(const DistillArgs a, int inner) {
    constexpr int N = Elem<DT>::N;
    extern __shared__ __align__(128) unsigned char ring[];
    __shared__ StreamBars bars;
    __shared__ __align__(16) Part s_part[kWarps];
    __shared__ Known s_known;
    __shared__ double s_red[kWarps][3];
    __shared__ unsigned s_outer;                 // which of the elements outside of the streamed part are the teacher's
    const int tid = threadIdx.x, lane = tid & 31, warp = warp_index();
    const unsigned row32 = blockIdx.x;
    const long long row = row32;
    const float w = a.weight ? a.weight[row] : 1.f;
    if (w == 0.f) {
        tell_nothing(a, row32);
        return;
    }
    int *ids = reinterpret_cast<int *>(ring + kMinStages * kTileBytes), *place = ids + (a.K + 3) / 4 * 4;
    float *xk = reinterpret_cast<float *>(place + (a.K + 4) / 4 * 4);
    const unsigned b = row32 / (unsigned)a.L, l = row32 - b * (unsigned)a.L;
    const DT *x = reinterpret_cast<const DT *>(a.x) + b * a.sb + l * a.sl;
    const int head = inner == a.V ? 0 : (int)((N - (reinterpret_cast<uintptr_t>(x) / sizeof(DT)) % N) % N);
    if (tid == 0) s_outer = 0u;
    stream_begin(bars, kMinStages);

    int id = -1, rank = -1;
    float outer_x = -CUDART_INF_F, x_mine = 0.f; // an element outside of the streamed part; the slot's token, if it is one of those
    double lp, pk, P;
    auto list = [&]() {
        float t = -CUDART_INF_F;
        const float t_lse = a.tlse ? a.tlse[row] : 0.f;
        if (tid < a.K) {
            id = a.id[row * a.K + tid];
            t = a.val[row * a.K + tid];
            const int n = a.count ? a.count[row] : a.K;
            if (tid >= n || id < 0 || id >= a.V) id = -1;
        }
        if (tid < a.V - inner) outer_x = Elem<DT>::load1(x + (tid < head ? tid : inner + tid));
        if (tid < (a.K + 3) / 4 * 4) ids[tid] = id;
        __syncthreads();
        probabilities(a, id, t, t_lse, ids, s_red, lp, pk, P);
        __syncthreads();
        const bool in = id >= head && id < head + inner;
        if (tid < (a.K + 3) / 4 * 4) ids[tid] = in ? id : 0x7FFFFFFF;
        if (id >= 0 && !in) {
            atomicOr(&s_outer, 1u << (id < head ? id : id - inner));
            x_mine = Elem<DT>::load1(x + id);
        }
        __syncthreads();
        if (in) {
            const int4 *all = reinterpret_cast<const int4 *>(ids);
            rank = 0;
            for (int j = 0; j * 4 < a.K; ++j) {
                const int4 o = all[j];
                rank += (o.x < id) + (o.y < id) + (o.z < id) + (o.w < id);
            }
            place[rank] = id - head;
        }
        const int used = __syncthreads_count(in);
        if (tid == 0) place[used] = 0x7FFFFFFF;
        __syncthreads();
    };
    LossPass<DT, decltype(list)> pass(list, place, xk, a.s);
    ColTop top;
    ColSums cs;
    stream_slice<DT, true>(x + head, 0, inner, kMinStages, bars, ring, top, cs, pass);
    if (id >= 0 && rank < 0) pass.add_token(x_mine);
    if (warp == 0) {                             // the elements outside of the streamed part
        const bool other = lane < a.V - inner && !(s_outer >> lane & 1u);
        const float c1 = fmaxf(max_of_warp(other ? outer_x * a.s : kLowest), pass.c);
        pass.S = pass.S != 0.f ? pass.S * ex2_approx(pass.c - c1) : 0.f;
        if (other) pass.S += ex2_approx(fmaf(outer_x, a.s, -c1));
        pass.c = c1;
    }
    Part part = {pass.c, sum_of_warp(pass.S), max_of_warp(pass.ct), 0.f};
    part.E = sum_of_warp(pass.E != 0.f ? pass.E * ex2_approx(pass.ct - part.ct) : 0.f);
    if (lane == 0) s_part[warp] = part;
    __syncthreads();
    if (warp == 0) {
        if (a.tlse)
            for (int i = 0; i * 32 < a.K; ++i) P += s_red[i][0];
        const Known kn = known_of(a, s_part, kWarps, P, a.tlse ? a.tlse[row] : 0.f, lost_if(bars.timed_out), lane);
        if (lane == 0) s_known = kn;
    }
    __syncthreads();
    const float xt = id < 0 ? 0.f : rank < 0 ? x_mine : xk[rank];
    if (a.state && id >= 0) {
        const float q = __fdividef(ex2_approx((float)((double)xt * (double)a.s - (double)s_known.c_all)), s_known.all);
        a.state[row * (a.K + 4) + 4 + tid] = s_known.none ? 0.f : (float)(((double)q - pk) * a.inv_t);
    }
    tell_row(a, row32, id, lp, pk, P, xt, s_known, s_red, kThreads);
    if (tid == 0 && bars.timed_out && a.status) atomicOr(&a.status[b], DSP_ROW_TIMEOUT);
}

// The gradient from what dsp_distill left of the row: c, f and the K elements.
struct DistillGradArgs {
    const void *x;
    long long sb, sl;
    int L, V, K, slices, per;                   // pieces of a slice
    const int32_t *id;
    const float *state, *factor;
    float s;
    void *g;
    long long gsb, gsl;
};
constexpr int kGradVecs = 2048;                 // 32 KB of a row for a CTA; 16 and 48 KB: the same within 1%

template <typename DT>
__global__ void __launch_bounds__(kDT) distill_grad_kernel(const DistillGradArgs a) {
    constexpr int N = Elem<DT>::N;
    extern __shared__ __align__(128) unsigned char ring[];
    __shared__ CopyBar sh;
    DT *buf = reinterpret_cast<DT *>(ring);
    const int tid = threadIdx.x;
    const unsigned row32 = blockIdx.x / (unsigned)a.slices, slice = blockIdx.x - row32 * (unsigned)a.slices;
    const unsigned b = row32 / (unsigned)a.L, l = row32 - b * (unsigned)a.L;
    const long long row = row32;
    const DT *x = reinterpret_cast<const DT *>(a.x) + b * a.sb + l * a.sl;
    DT *g = reinterpret_cast<DT *>(a.g) + b * a.gsb + l * a.gsl;
    const Pieces<DT> p(x, a.V);
    const int p0 = (int)min(slice * (unsigned)a.per, (unsigned)p.n), p1 = (int)min((slice + 1) * (unsigned)a.per, (unsigned)p.n);
    const float *state = a.state + row * (a.K + 4);
    const float w = a.factor[row], c = state[0], f = state[1];
    // the slot's own element, if it lies in this slice (-1: none), and its gradient
    int at = -1;
    float gk = 0.f;
    auto own = [&]() {
        if (tid >= a.K || __float_as_uint(state[4 + tid]) == kNoEntry) return;
        const int id = a.id[row * a.K + tid];
        if (id < 0 || id >= a.V) return;
        const int piece = (p.h + id) / N;
        if (piece < p0 || piece >= p1) return;
        at = id;
        gk = state[4 + tid] * w;
    };
    if (w == 0.f || f == 0.f) {                 // nothing for the others, whatever their logits are: dsp_distill may not have read them either
        if (w != 0.f) own();
        store_zeros<DT>(g, max(0, p0 * N - p.h), min(a.V, p1 * N - p.h));
        __syncthreads();
        if (at >= 0) g[at] = rounded<DT>(gk);
        return;
    }
    if (tid == 0) {
        mbar_init(&sh.bar, 1);
        mbar_init_fence();
        sh.timed_out = 0;
    }
    __syncthreads();
    if (tid == 0) send_copies<DT>(x, p, p0, p1, buf, sh);
    read_edges<DT>(x, p, a.V, p0, p1, buf);
    own();
    if (tid < 32) take_copies(sh, 0u);
    __syncthreads();
    write_pieces<DT>(g, p, a.V, p0, p1, buf, a.s, c, sh.timed_out ? CUDART_NAN_F : f * w);
    __syncthreads();                            // the token's own element comes after the piece that it lies in
    if (at >= 0) g[at] = rounded<DT>(gk);
}

inline int pieces_at_most(int V, int N) { return (int)(((long long)V + 2 * N - 2) / N); }

constexpr int kMaxBufVecs = 216 * 1024 / 16;

template <typename DT, bool GRAD, int CTAS>
int32_t launch_distill_rows(const DistillArgs &a, long long rows, cudaStream_t st) {
    static std::atomic<unsigned long long> smem_done{0};
    DSP_CUDA_TRY(allow_shared(distill_kernel<DT, GRAD, CTAS>, kMaxBufVecs * 16, smem_done));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(rows * a.C));
    cfg.blockDim = dim3(kDT);
    cfg.dynamicSmemBytes = (size_t)a.buf_vecs * 16;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)a.C;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = a.C > 1 ? 1 : 0;
    DSP_CUDA_TRY(cudaLaunchKernelEx(&cfg, distill_kernel<DT, GRAD, CTAS>, a));
    DSP_CUDA_TRY(cudaGetLastError());
    return DSP_OK;
}

template <typename DT, bool GRAD>
int32_t launch_distill(DistillArgs &a, long long rows, cudaStream_t st) {
    constexpr int N = Elem<DT>::N;
    const int n = pieces_at_most(a.V, N);
    int C = 1;
    while (C < kMaxCluster && (long long)n > (long long)C * kSliceVecs) C *= 2;
    // Few rows are cut finer, as long as a thread keeps a piece (us, without / with): 100 rows of 64000 bf16 10.3 / 9.6, 40 of 32003 fp32
    // 7.2 / 7.1; up to three CTAs an SM instead of two: 100 rows of 32000 10.9 / 7.4, of 64000 12.6 / 9.6.
    while (C < kMaxCluster && rows * C < 2 * device_sm_count() && n >= 2 * C * kDT) C *= 2;
    a.C = C;
    while ((1 << a.log2_c) < C) ++a.log2_c;
    const int per = (n + C - 1) / C;
    a.buf_vecs = per < kMaxBufVecs ? per : kMaxBufVecs;
    if (rows * C > 0x7FFFFFFFLL) return DSP_ERR_UNSUPPORTED;
    // Five CTAs an SM where their buffers fit and there are as many, else four, with more registers.  Measured (us, five / four): 2048 rows of
    // 152064 bf16 225 / 245, with K = 256 278 / 311; 1000 of 100000 76.8 / 75.5, of 32000 30.4 / 30.1, 999 of 32003 fp32 49.8 / 49.2, whose buffers let three fit.
    if (a.buf_vecs <= 2560 && rows * C > 4 * device_sm_count()) return launch_distill_rows<DT, GRAD, 5>(a, rows, st);
    return launch_distill_rows<DT, GRAD, 4>(a, rows, st);
}

constexpr int kLongRow = 75000;                 // logits from which a row is streamed for its loss: see dsp_distill's dispatch
int32_t launch_distill_loss(const DistillArgs &a, long long rows, cudaStream_t st) {
    using DT = __nv_bfloat16;
    constexpr int N = Elem<DT>::N;
    // elements of a row that are streamed: all of it where every row starts on 16 bytes, else the pieces that lie inside it at any start
    const int inner = stream_layout_ok<DT>(a.x, a.V, a.sb, a.sl) ? a.V : (a.V - (N - 1)) / N * N;
    static std::atomic<unsigned long long> smem_done{0};
    DSP_CUDA_TRY(allow_shared(distill_loss_kernel<DT>, kMinStages * kTileBytes + loss_list_words(DSP_MAX_TEACHER) * 4, smem_done));
    distill_loss_kernel<DT><<<(unsigned)rows, kThreads, (size_t)(kMinStages * kTileBytes + loss_list_words(a.K) * 4), st>>>(a, inner);
    DSP_CUDA_TRY(cudaGetLastError());
    return DSP_OK;
}

template <typename DT>
int32_t launch_distill_grad(DistillGradArgs &a, long long rows, cudaStream_t st) {
    const int n = pieces_at_most(a.V, Elem<DT>::N);
    a.slices = (n + kGradVecs - 1) / kGradVecs;
    if (rows * a.slices > 0x7FFFFFFFLL) return DSP_ERR_UNSUPPORTED;
    a.per = (n + a.slices - 1) / a.slices;
    distill_grad_kernel<DT><<<(unsigned)(rows * a.slices), kDT, (size_t)a.per * 16, st>>>(a);
    DSP_CUDA_TRY(cudaGetLastError());
    return DSP_OK;
}

int32_t check_rows(int32_t dtype, int32_t B, int32_t L, int32_t V, int32_t K, float temperature) {
    if (B < 0 || L < 1 || V < 1 || K < 1 || !(temperature >= 1e-3f && temperature <= 1e3f)) return DSP_ERR_INVALID_ARG;
    if ((dtype != DSP_F32 && dtype != DSP_BF16) || K > DSP_MAX_TEACHER || V > (1 << 30) || (long long)B * L > (1 << 24))
        return DSP_ERR_UNSUPPORTED;
    return DSP_OK;
}
bool rows_fit(const void *p, size_t es, int64_t sb, int64_t sl, int32_t B, int32_t L, int32_t V) {
    if ((reinterpret_cast<uintptr_t>(p) & (es - 1)) != 0 || sl < V || sb < 0) return false;
    return B == 1 || sb >= (int64_t)(L - 1) * sl + V;
}

}  // namespace
}  // namespace dsp

extern "C" int32_t dsp_distill(const void *student_logits, int32_t dtype, int32_t B, int32_t L, int32_t V,
                               int64_t stride_b, int64_t stride_l, const int32_t *teacher_id, const float *teacher_logit,
                               const float *teacher_lse, const int32_t *teacher_count, int32_t K, float temperature,
                               const float *weight, float *loss, float *accept, float *lse, float *state,
                               void *grad, int64_t grad_stride_b, int64_t grad_stride_l,
                               uint32_t *row_status, dsp_stream_t stream) {
    using namespace dsp;
    const int32_t rc = check_rows(dtype, B, L, V, K, temperature);
    if (rc != DSP_OK) return rc;
    if (B == 0) return DSP_OK;
    const size_t es = dtype == DSP_BF16 ? 2 : 4;
    if (!student_logits || !teacher_id || !teacher_logit || !loss) return DSP_ERR_INVALID_ARG;
    if (!rows_fit(student_logits, es, stride_b, stride_l, B, L, V)) return DSP_ERR_INVALID_ARG;
    if (grad && !rows_fit(grad, es, grad_stride_b, grad_stride_l, B, L, V)) return DSP_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(state) & 15) != 0) return DSP_ERR_INVALID_ARG;
    DistillArgs a = {};
    a.x = student_logits; a.sb = stride_b; a.sl = stride_l;
    a.L = L; a.V = V; a.K = K;
    a.id = teacher_id; a.count = teacher_count; a.val = teacher_logit; a.tlse = teacher_lse; a.weight = weight;
    a.inv_t = 1.0 / (double)temperature;
    a.s = (float)(a.inv_t / kLn2);
    a.inv_s = a.inv_t / (double)a.s;
    a.loss = loss; a.accept = accept; a.lse = lse; a.state = state;
    a.g = grad; a.gsb = grad_stride_b; a.gsl = grad_stride_l;
    a.status = row_status;
    const long long rows = (long long)B * L;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    // The loss alone of many long bf16 rows streams each in a CTA; measured with the gradient's call behind it, K = 16 (us, streamed / by
    // clusters): 512 rows of 152064 90 / 95, 148 rows 32.3 / 32.3, 32 rows 22 / 13; 600 rows of 100000 76 / 73, of 200000 131 / 133, of 64000 57 / 50;
    // 2000 rows of 110000 225 / 248, of 80000 179 / 179; fp32 (half the logits for the same bytes, the same work a tile) 600 rows of 100000 152 / 127.
    // By clusters, both calls: 600 rows of 64000 bf16 50, fp32 86, 2000 of 32003 fp32 140; streamed with K = 256: 512 rows of 152064 153.
    if (!grad && dtype == DSP_BF16 && rows >= device_sm_count() && V >= kLongRow) return launch_distill_loss(a, rows, st);
    if (dtype == DSP_BF16)
        return grad ? launch_distill<__nv_bfloat16, true>(a, rows, st) : launch_distill<__nv_bfloat16, false>(a, rows, st);
    return grad ? launch_distill<float, true>(a, rows, st) : launch_distill<float, false>(a, rows, st);
}

extern "C" int32_t dsp_distill_grad(const void *student_logits, int32_t dtype, int32_t B, int32_t L, int32_t V,
                                    int64_t stride_b, int64_t stride_l, const int32_t *teacher_id, int32_t K,
                                    const float *state, float temperature, const float *row_grad,
                                    void *grad, int64_t grad_stride_b, int64_t grad_stride_l, dsp_stream_t stream) {
    using namespace dsp;
    const int32_t rc = check_rows(dtype, B, L, V, K, temperature);
    if (rc != DSP_OK) return rc;
    if (B == 0) return DSP_OK;
    const size_t es = dtype == DSP_BF16 ? 2 : 4;
    if (!student_logits || !teacher_id || !state || !row_grad || !grad) return DSP_ERR_INVALID_ARG;
    if (!rows_fit(student_logits, es, stride_b, stride_l, B, L, V) || !rows_fit(grad, es, grad_stride_b, grad_stride_l, B, L, V))
        return DSP_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(state) & 15) != 0) return DSP_ERR_INVALID_ARG;
    DistillGradArgs a = {};
    a.x = student_logits; a.sb = stride_b; a.sl = stride_l;
    a.L = L; a.V = V; a.K = K;
    a.id = teacher_id; a.state = state; a.factor = row_grad;
    a.s = (float)(1.0 / (double)temperature / kLn2);
    a.g = grad; a.gsb = grad_stride_b; a.gsl = grad_stride_l;
    const long long rows = (long long)B * L;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    return dtype == DSP_BF16 ? launch_distill_grad<__nv_bfloat16>(a, rows, st) : launch_distill_grad<float>(a, rows, st);
}
