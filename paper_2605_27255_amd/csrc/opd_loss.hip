// OPD losses with their gradients (App. C): the divergence of a student row
// from a teacher's top logits, and the clipped policy loss of a row's label.
//
// With x = z / temperature, both are functions of the log-probabilities of a
// few listed entries of the row (the teacher's ids; the label) and of the mass
// of all others.  For a = p df/dp of each entry and of the rest r, A = sum a:
//   dL/dz_v = (a_v - p_v A) / temperature                       v listed
//   dL/dz_v = (a_r softmax_rest(v) - p_v A) / temperature        v not listed
// so the row's gradient away from the list is exp((z_v - m) / temperature)
// times one number.  One pass over the row gives the sum of exponentials of the
// unlisted values over a reference (a bitmap of the listed ids in LDS drops them
// from the sum, so the rest's mass carries no cancellation even where it is
// tiny); everything per entry is 64-bit arithmetic on a handful of numbers; a
// second pass, from registers and LDS as far as the row fits, writes the
// gradient, and the listed entries are written over it.
// HBM-bound: V logits read, V gradients written.  2048 x 151936 with the
// gradient, a tenth of the positions not scored and only written: bf16 248 us, 4.8
// TB/s (a copy of as many bytes: 224 us), fp32 488 us, 4.8 TB/s (478 us); without
// the gradient bf16 99 us, 6.3 TB/s, fp32 184 us, 6.8 TB/s.
//
// Where there are too few rows for the chip, each is split over several
// workgroups: k_opd_part sums a segment and gathers the listed logits,
// k_opd_apply joins the segments' sums (every workgroup for itself, from a few
// numbers) and writes its segment's gradient.
#include "opd_rows.h"
#include "pipo.h"

namespace pipo {

constexpr int kEntries = 256;       // listed entries of a row
constexpr size_t kLdsBytes = 160 * 1024;
constexpr int kOpdMaxRows = (1 << 22) - 1;      // threads of a launch are counted in 32 bits
constexpr int64_t kOpdMaxStride = (int64_t)1 << 31;

template <typename L> struct LossParams {
    const L *z; int64_t ld;
    int T, V;
    int kind;                       // PIPO_OPD_* or kPolicy
    ExpScale c;
    double beta;
    // distillation
    int Tt, k;
    const int32_t *ids; const float *q, *q_rest; const int32_t *rows;
    // policy
    const float *adv, *old_lp, *ref_lp;
    double clip_lo, clip_hi, kl_coef;
    const int32_t *labels;
    const float *scale;
    float *loss, *logp, *kl;
    L *grad; int64_t ldg;
    int pieces;                     // whole pieces that every row has
    int spill;                      // slabs of a row in LDS, behind those in registers
};
constexpr int kPolicy = 3;

struct LossShared {
    int id[kEntries];               // listed ids, -1: an empty slot
    float z[kEntries], q[kEntries];     // their logits, the teacher's log-probabilities
    double a[kEntries], p[kEntries];   // their a = p df/dp, and p
    float patch[kEntries];          // their gradients
    float coef, B;                  // the others' gradient over 2^(z c - B)
    int bad;
};

// What happens at position t: not scored, flagged (no such row, label or id), or scored with k entries.
enum { kSkip, kFlag, kScore };

// Position t's own numbers (the same for the whole workgroup: scalar loads).
struct Position {
    int what, y, trow;
    float scale, q_rest, adv, old_lp, ref_lp;
};
template <typename L> __device__ __forceinline__ Position read_position(const LossParams<L> &p, int t) {
    Position x;
    x.y = p.labels ? p.labels[t] : 0;
    x.trow = p.rows ? p.rows[t] : t;
    x.scale = p.scale ? p.scale[t] : 1.f;
    x.q_rest = x.adv = x.old_lp = x.ref_lp = 0.f;
    if (p.kind == kPolicy) {
        x.adv = p.adv[t];
        if (p.old_lp) x.old_lp = p.old_lp[t];
        if (p.ref_lp) x.ref_lp = p.ref_lp[t];
        x.what = x.y < 0 ? kSkip : x.y >= p.V ? kFlag : kScore;
    } else {
        x.what = x.y < 0 ? kSkip : x.trow < 0 || x.trow >= p.Tt ? kFlag : kScore;
        if (p.q_rest && x.what == kScore) x.q_rest = p.q_rest[x.trow];
    }
    return x;
}
// Entry j of a scored position: its id and the teacher's log-probability.
template <typename L>
__device__ __forceinline__ void read_entry(const LossParams<L> &p, int j, const Position &x, int &id, float &q) {
    id = -1;
    q = 0.f;
    if (j >= p.k || x.what != kScore) return;
    if (p.kind == kPolicy) {
        id = x.y;
    } else {
        id = p.ids[(int64_t)x.trow * p.k + j];
        q = p.q[(int64_t)x.trow * p.k + j];
    }
}
// A bit of the bitmap for each element of a row's (or segment's) pieces, the
// partial piece -1 first: element `at` has bit at - head + N.
template <typename L> __host__ __device__ __forceinline__ int bitmap_words(int n) { return (n + 2 * Piece<L>::N + 127) / 128 * 4; }
// Marks the listed ids of the segment [lo, lo + row.n) in a cleared bitmap and
// keeps all entries in LDS; sh.bad, cleared before, is set where one is out of
// range, or twice in this segment.  Thread j brings entry j.
template <typename L>
__device__ __forceinline__ void mark_entry(int id, float q, int k, int V, int lo, const Span<L> &row, LossShared &sh, uint32_t *bits) {
    const int tid = threadIdx.x;
    if (tid >= k) return;
    sh.id[tid] = id;
    sh.q[tid] = q;
    const int at = id - lo, bit = at - row.head + 16 / (int)sizeof(L);
    if (id >= V || (id >= lo && at < row.n && (atomicOr(&bits[bit >> 5], 1u << (bit & 31)) >> (bit & 31) & 1u))) sh.bad = 1;
}
template <int NT> __device__ __forceinline__ void clear_bits(uint32_t *bits, int words, LossShared &sh) {
    for (int i = threadIdx.x; i < words; i += NT) bits[i] = 0;
    if (threadIdx.x == 0) sh.bad = 0;
}

// The bitmap's bits of piece i (bit e: its element e is listed).
template <int N> __device__ __forceinline__ uint32_t listed_bits(const uint32_t *bits, int i) {
    const uint32_t b = ((const uint8_t *)bits)[(i + 1) * N >> 3];
    return N == 8 ? b : (b >> (((i + 1) & 1) * 4)) & 15u;
}

// One entry's share of a divergence and a = p df/dp, from the student's and the teacher's log-probabilities.
__device__ __forceinline__ void divergence(int kind, double beta, double lp, double lq, double &f, double &a) {
    const double p = exp(lp), q = exp(lq);
    if (kind == PIPO_OPD_FORWARD) {
        f = q == 0. ? 0. : q * (lq - lp);
        a = -q;
        if (lp != lp) f = a = lp;
    } else if (kind == PIPO_OPD_REVERSE) {
        f = p == 0. ? 0. : p * (lp - lq);
        a = f + p;
    } else {
        const double lm = log(beta * q + (1. - beta) * p);
        const double pl = p == 0. ? 0. : p * (lp - lm);
        f = beta * (q == 0. ? 0. : q * (lq - lm)) + (1. - beta) * pl;
        a = (1. - beta) * pl;
    }
}

// The first wave turns the listed logits and the rest's (max, sum) into the
// position's outputs (where `first`) and its gradient's numbers; ends with a barrier.
template <typename L>
__device__ __forceinline__ void finish_row(const LossParams<L> &p, int t, const Position &x, RowSum rest, LossShared &sh,
                                           bool first = true) {
    if (threadIdx.x < 64) {
        const int lane = threadIdx.x;
        const double inv = p.c.inv;
        float top = rest.m;
        for (int j = lane; j < p.k; j += 64) if (sh.id[j] >= 0) top = fmaxf(top, sh.z[j]);
        const double m = wave_max_dpp(top);
        double sum = 0.;
        for (int j = lane; j < p.k; j += 64) if (sh.id[j] >= 0) sum += exp(((double)sh.z[j] - m) * inv);
        sum = wave_sum_f64(sum);
        const double unit = log_unit(rest.m, rest.B, m, p.c);
        const double rest_at = rest.m == -INFINITY ? 1. : exp(unit);
        // without a rest its sum is 0 (or NaN); one that nearly vanishes beside the list: what the sum's rounding takes goes
        // into the log
        const double x_rest = rest.s * rest_at, whole = sum + x_rest, lost = x_rest <= sum ? x_rest - (whole - sum) : 0.;
        // of x - m / temperature; a row without any mass has none
        const double lse = m == -INFINITY ? (double)__builtin_nanf("") : log(whole) + lost;
        const double g = (double)x.scale * inv;
        double A = 0., a_rest = 0.;
        if (p.kind == kPolicy) {
            const double lp = ((double)sh.z[0] - m) * inv - lse, adv = x.adv;
            const double r = p.old_lp ? exp(lp - (double)x.old_lp) : lp == lp ? 1. : lp;     // on-policy: 1 for a masked label too
            const double cut = fmin(fmax(r, 1. - p.clip_lo), 1. + p.clip_hi);
            const bool inside = adv * r <= adv * cut;
            double loss = -(inside ? adv * r : adv * cut), d = inside ? -adv * r : 0., kl = 0.;
            if (r != r || adv != adv) loss = d = r + adv;
            if (p.ref_lp) {
                const double far = (double)x.ref_lp - lp;
                kl = far == INFINITY ? far : expm1(far) - far;
                if (p.kl_coef != 0.) {
                    loss += p.kl_coef * kl;
                    d -= p.kl_coef * expm1(far);
                }
            }
            A = d;
            if (lane == 0 && first) {
                p.loss[t] = (float)loss;
                if (p.logp) p.logp[t] = (float)lp;
                if (p.kl) p.kl[t] = (float)kl;
            }
        } else {
            double f = 0.;
            // entry k stands for the tokens outside the list
            for (int j = lane; j < p.k + (p.q_rest ? 1 : 0); j += 64) {
                const bool out = j == p.k;
                if (!out && sh.id[j] < 0) continue;
                double lp = out ? unit + log(rest.s) - lse : ((double)sh.z[j] - m) * inv - lse;
                if (out && rest.s == 0.) lp = lse == lse ? -INFINITY : lse;
                double fj, aj;
                divergence(p.kind, p.beta, lp, out ? (double)x.q_rest : (double)sh.q[j], fj, aj);
                f += fj;
                A += aj;
                if (out) a_rest = aj;
                else { sh.a[j] = aj; sh.p[j] = exp(lp); }
            }
            f = wave_sum_f64(f);
            A = wave_sum_f64(A);
            a_rest = readlane_f64(a_rest, p.k & 63);
            if (!(lse == lse)) f = lse;
            if (lane == 0 && first) p.loss[t] = (float)f;
            if (p.grad) {
                for (int j = lane; j < p.k; j += 64)
                    if (sh.id[j] >= 0) sh.patch[j] = (float)(g * (sh.a[j] - sh.p[j] * A));
            }
        }
        if (lane == 0 && p.grad) {
            const double unit_p = rest_at * exp(-lse);      // the probability of one of the rest's units
            if (p.kind == kPolicy) sh.patch[0] = (float)(g * A * (rest.s * unit_p));    // (1 - p of the label without cancellation)
            // with no mass outside the list there is nothing to spread there
            const double k = lse != lse ? lse : rest.s == 0. ? 0. : g * (a_rest / rest.s - A * unit_p);
            // against a reference near the values that weigh most: their exponents are small, and so their roundings
            // (k counts from the one that a float holds, which far from 0 is not the sum's plus a whole number)
            const int shift = is_far(rest.m, p.c) || !(rest.s > 0.) ? 0 : min(max(ilogb(rest.s), -120), 120);
            const float B = rest.B + (float)shift;
            const double off = (double)B - (double)rest.B;
            sh.coef = (float)(off == (double)shift ? ldexp(k, shift) : k * exp2(off));
            sh.B = B;
        }
    }
    __syncthreads();
}

template <typename L, int NT>
__device__ __forceinline__ void fill_row(L *row, int n, float v) {
    const Span<L> to(row, n);
    float x[Piece<L>::N];
#pragma unroll
    for (int e = 0; e < Piece<L>::N; ++e) x[e] = v;
    for (int i = threadIdx.x; i < to.whole; i += NT) store_piece(to.body, i, x);
    if (!to.exact() && (int)threadIdx.x >= NT - 2) store_edge(to.body, to, (int)threadIdx.x == NT - 1 ? -1 : to.whole, x);
}

// A position that is not scored (zeros) or flagged (NaN).
template <typename L>
__device__ __forceinline__ void put_constant(const LossParams<L> &p, int t, float v) {
    if (threadIdx.x != 0) return;
    p.loss[t] = v;
    if (p.logp) p.logp[t] = v;
    if (p.kl) p.kl[t] = v;
}

// A piece of a row (or segment) into a sum, without its listed elements.
template <typename L>
__device__ __forceinline__ void add_piece(MaxSum<double> &a, u32x4 w, int i, const uint32_t *bits, ExpScale c) {
    constexpr int N = Piece<L>::N;
    const uint32_t b = listed_bits<N>(bits, i);
    float v[N];
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = Piece<L>::get(w, e);
    if (b) {
#pragma unroll
        for (int e = 0; e < N; ++e) if (b >> e & 1u) v[e] = -INFINITY;
    }
    add_values<N>(a, v, c);
}
// The sum of a row (or segment) of far values, by differences from its maximum m.
template <typename L, int NT>
__device__ __forceinline__ double sum_far(const Span<const L> &row, const uint32_t *bits, float m, ExpScale c, double *s_w) {
    constexpr int N = Piece<L>::N;
    float s = 0.f;
    each_piece<NT, 1>(row, (int)threadIdx.x, [&](u32x4 w, int i) {
        const uint32_t b = listed_bits<N>(bits, i);
#pragma unroll
        for (int e = 0; e < N; ++e) if (!(b >> e & 1u)) s += exp_diff(Piece<L>::get(w, e), m, c);
    });
    return block_sum<NT>(s, s_w);
}
// A piece's gradients away from the list; those of listed elements are written over them later.
template <typename L> __device__ __forceinline__ void gradients(float *v, u32x4 w, float coef, float B, ExpScale c) {
    // with c's second float, as in the sum: z times it is no rounding, but a tilt of the whole row (1e-4 at z = 1000 and
    // temperature 0.7), which the exponents, differences that they are, would not show
#pragma unroll
    for (int e = 0; e < Piece<L>::N; ++e) v[e] = coef * exp_at(Piece<L>::get(w, e), B, c);
}
// ... of this thread's pieces from index first on, and the partial ones (out: where the gradient's piece 0 lies).
template <typename L, int NT>
__device__ __forceinline__ void put_pieces(L *out, const Span<const L> &row, int first, float coef, float B, ExpScale c) {
    whole_pieces<NT, 4, true>(row.body, first, row.whole, [&](u32x4 w, int i) {
        float v[Piece<L>::N];
        gradients<L>(v, w, coef, B, c);
        store_piece(out, i, v);
    });
    edges<NT>(row, [&](u32x4 w, int i) {
        float v[Piece<L>::N];
        gradients<L>(v, w, coef, B, c);
        store_edge(out, row, i, v);
    });
}
template <typename L, int NT>
__device__ __forceinline__ void put_far(L *out, const Span<const L> &row, float coef, float m, ExpScale c) {
    constexpr int N = Piece<L>::N;
    each_piece<NT, 1>(row, (int)threadIdx.x, [&](u32x4 w, int i) {
        float v[N];
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = coef * exp_diff(Piece<L>::get(w, e), m, c);
        if (i >= 0 && i < row.whole) store_piece(out, i, v);
        else store_edge(out, row, i, v);
    });
}

// A thread's sum of 2^(z c - B), and its largest piece's share and slab.
struct PieceSum { double s; float most; int slab; };
// Adds a piece, unless it holds a listed element.
template <typename L> __device__ __forceinline__ void sum_piece(PieceSum &a, u32x4 w, int slab, uint32_t listed, float B, ExpScale c) {
    constexpr int N = Piece<L>::N;
    float x = 0.f;
#pragma unroll
    for (int e = 0; e < N; ++e) x += exp_at(Piece<L>::get(w, e), B, c);
    x = listed ? 0.f : x;
    a.s += x;
    if (x > a.most) { a.most = x; a.slab = slab; }
}
// Values far above the reference have large exponents, whose rounding the sum
// would show: what it cost in this piece.
template <typename L> __device__ __forceinline__ float rounding_of(u32x4 w, float B, ExpScale c) {
    float x = 0.f;
#pragma unroll
    for (int e = 0; e < Piece<L>::N; ++e) {
        const float z = Piece<L>::get(w, e), r = fmaf(z, c.lo, fmaf(z, c.hi, -B)), term = __builtin_amdgcn_exp2f(r);
        const double off = fma((double)z, (double)c.lo, fma((double)z, (double)c.hi, -(double)B)) - (double)r;
        if (term > 0.f) x = fmaf(term * (float)kLn2, (float)off, x);
    }
    return x;
}
template <typename L> __device__ __forceinline__ void max_piece(float &m, u32x4 w, uint32_t listed) {
    constexpr int N = Piece<L>::N;
    float x = Piece<L>::get(w, 0);
#pragma unroll
    for (int e = 1; e < N; ++e) x = fmaxf(x, Piece<L>::get(w, e));
    m = fmaxf(m, listed ? -INFINITY : x);
}
// (max, sum) of the unlisted elements of a row where the reference of the fast
// pass did not fit, from two passes of their own.
template <typename L, int NT>
__device__ __forceinline__ RowSum sum_slowly(const Span<const L> &row, const uint32_t *bits, ExpScale c, Reduce<NT> &red) {
    MaxSum<double> own{-INFINITY, 0.};
    each_piece<NT, 1>(row, (int)threadIdx.x, [&](u32x4 w, int i) { add_piece<L>(own, w, i, bits, c); });
    __syncthreads();
    RowSum a = block_merge<NT>(own, c, red);
    __syncthreads();
    if (is_far(a.m, c)) a.s = sum_far<L, NT>(row, bits, a.m, c, red.sum[1]);
    __syncthreads();
    return a;
}

// A workgroup takes positions blockIdx.x, + gridDim.x, ...  Of a row's whole
// slabs (a piece for every thread) the first NV stay in registers between the two
// passes; what lies behind them is read again.
//   The sum's reference is the largest unlisted value of the first AHEAD slabs
// (where masks hide all of them, the largest listed one), which a row's maximum
// does not pass by more than a float holds (2^127) in earnest; a row that does has
// an infinite sum (or, masked, next to none), and is summed again slowly.  So no
// value needs a comparison, and no sum is rescaled.  Pieces with a listed element
// are left out and added by the thread that brings the entry.
// (A row longer than the most slabs that registers hold keeps some in LDS.)
//   Rows that run with NV slabs have at least NV - STEP of them.
//   The AHEAD slabs are loaded while the position before is written, the others
// AHEAD slabs before their sum, so that neither loads nor sums wait for all of
// the other.
template <int NT, int NV> constexpr bool kTakesSeveral = NT == 512 && NV >= 12;    // one workgroup fills a compute unit
template <int NT, int NV> constexpr bool kSpills = NV >= (NT == 512 ? 32 : 44);     // the longest rows' variants
// Waves of a SIMD that the registers leave room for: short rows live by their number (16384 x 8192 bf16 with the gradient
// from five 108 us, from six 99).  Workgroups of sixteen waves have a compute unit to themselves.
constexpr int waves_of(int nt, int nv, bool grad) { return !grad ? (nt == 1024 ? 4 : 8) : nv <= 2 ? 7 : nv <= 4 ? 6 : nv <= 8 ? 5 : nt / 256; }
template <typename L, int NT, int NV, int STEP, bool GRAD>
__global__ __launch_bounds__(NT, waves_of(NT, NV, GRAD)) void k_opd_loss(LossParams<L> p) {
    constexpr bool LOOP = kTakesSeveral<NT, NV>, DEEP = kSpills<NT, NV>;
    constexpr int AHEAD = NV < 12 ? NV : 12, N = Piece<L>::N;
    extern __shared__ uint32_t bits[];
    __shared__ LossShared sh;
    __shared__ Reduce<NT> red;
    const int tid = threadIdx.x, V = p.V;
    const int held = min(NV, p.pieces / NT), lower = DEEP ? held + p.spill : held;
    u32x4 *more = (u32x4 *)(bits + bitmap_words<L>(V));
    auto has = [&](int j) { return j < NV - STEP || j < held; };
    // the bitmap's bits of this thread's piece in slab j: a constant number of bytes further for each slab
    const uint8_t *bits0 = (const uint8_t *)bits + ((tid + 1) * N >> 3);
    const int shift0 = N == 8 ? 0 : ((tid + 1) & 1) * 4;
    auto listed = [&](int j) { return ((uint32_t)bits0[j * (NT * N / 8)] >> shift0) & (N == 8 ? 255u : 15u); };
    // Slab j's piece.  One that is not wanted comes from the row's first bytes: a branch around each load would
    // double the registers it is loaded into.  (Rows of less than a slab may not have those.)
    auto slab = [&](const L *from, int j, uint32_t off, bool wanted) {
        if (NV > STEP) return load_at(from, wanted && has(j) ? off : 0);
        return wanted && has(j) ? load_at(from, off) : u32x4{0, 0, 0, 0};
    };
    u32x4 keep[NV];
    int t = blockIdx.x, id;
    float q;
    Position x = read_position(p, t);
    Span<const L> row(p.z + (int64_t)t * p.ld, V);
    read_entry(p, tid, x, id, q);
    uint32_t off = tid * 16;
#pragma unroll
    for (int j = 0; j < AHEAD; ++j, next_slab<NT>(off)) keep[j] = slab(row.body, j, off, x.what == kScore);
    clear_bits<NT>(bits, bitmap_words<L>(V), sh);
    __syncthreads();
    for (;;) {
        const int next = t + gridDim.x;
        Position nx;
        nx.what = kSkip;
        if (LOOP && next < p.T) nx = read_position(p, next);
        L *out = GRAD ? p.grad + (int64_t)t * p.ldg : nullptr;
        bool scored = x.what == kScore, far = false;
        if (scored) {
            mark_entry(id, q, p.k, V, 0, row, sh, bits);
            __syncthreads();
            scored = sh.bad == 0;
        }
        RowSum a{-INFINITY, 0.f, 0.};
        if (scored) {
            // this thread's entry: its logit and, if it is the first listed one of its piece, the piece's others
            float zj = 0.f;
            PieceSum sum{0., 8.f, -1};
            u32x4 shared_piece;
            uint32_t others = 0;
            if (id >= 0) {
                zj = Piece<L>::one(row.body + (id - row.head));
                const int i = (id - row.head + N) / N - 1, e = (id - row.head + N) % N;
                const uint32_t here = listed_bits<N>(bits, i);
                if ((here & ((1u << e) - 1)) == 0) {
                    others = ~here;
                    shared_piece = i >= 0 && i < row.whole ? load_piece(row.body, i) : load_edge(row, i);
                }
            }
            float m = -INFINITY;
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                if (has(j)) max_piece<L>(m, keep[j], listed(j));
                __builtin_amdgcn_sched_barrier(0);
            }
            if (NV <= STEP && held == 0) each_piece<NT, 1>(row, tid, [&](u32x4 w, int i) { max_piece<L>(m, w, listed_bits<N>(bits, i)); });
            m = block_max<NT>(m, red.max[0]);
            const bool borrowed = !(m * p.c.hi > -kFar);
            if (borrowed) m = block_max<NT>(id >= 0 ? zj : -INFINITY, red.max[1]);
            const float B = ref_of(m, p.c);
            off = (tid + NT * AHEAD) * 16;
#pragma unroll
            for (int j = 0; j < NV; ++j, next_slab<NT>(off)) {
                if (j + AHEAD < NV) keep[j + AHEAD] = slab(row.body, j + AHEAD, off, true);
                asm volatile("" : "+v"(keep[j]));   // unpacked again: the floats would take twice the registers
                if (has(j)) sum_piece<L>(sum, keep[j], j, listed(j), B, p.c);
            }
            if (DEEP)
                whole_pieces<NT, 4>(row.body, tid + NT * held, NT * lower, [&](u32x4 w, int i) {
                    more[i - NT * held] = w;
                    sum_piece<L>(sum, w, i / NT, listed_bits<N>(bits, i), B, p.c);
                });
            whole_pieces<NT, 4, GRAD>(row.body, tid + NT * lower, row.whole, [&](u32x4 w, int i) {
                sum_piece<L>(sum, w, i / NT, listed_bits<N>(bits, i), B, p.c);
            });
            double s = sum.s;
            if (sum.slab >= 0) s += rounding_of<L>(load_piece(row.body, tid + NT * sum.slab), B, p.c);
            edges<NT>(row, [&](u32x4 w, int i) {
                PieceSum edge{0., 8.f, -1};
                sum_piece<L>(edge, w, 0, listed_bits<N>(bits, i), B, p.c);
                s += edge.s;
            });
            if (others) {
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if (others >> e & 1u) s += exp_at(Piece<L>::get(shared_piece, e), B, p.c);
            }
            if (tid < p.k) sh.z[tid] = zj;
            a = RowSum{m, B, block_sum<NT>(s, red.sum[0])};
            if (!(a.s < INFINITY) || is_far(m, p.c) || (borrowed && (a.s < 1e-30 || m == -INFINITY))) a = sum_slowly<L, NT>(row, bits, p.c, red);
            far = is_far(a.m, p.c);
            if (id >= 0) bits[(id - row.head + N) >> 5] = 0;     // every wave is past its sums: ready for the next position
            finish_row(p, t, x, a, sh);
        } else {
            const float v = x.what == kSkip ? 0.f : __builtin_nanf("");
            put_constant(p, t, v);
            if (GRAD) fill_row<L, NT>(out, V, v);
            if (LOOP && x.what == kScore) {      // flagged by its list
                __syncthreads();
                clear_bits<NT>(bits, bitmap_words<L>(V), sh);
            }
        }
        const int mine = scored ? id : -1;
        const Span<const L> next_row(p.z + (int64_t)(nx.what == kScore ? next : t) * p.ld, V);
        read_entry(p, tid, nx, id, q);
        if (GRAD) {
            const float coef = sh.coef, B = sh.B;
            const bool put = scored && !far;
            L *body = out + row.head;
            off = tid * 16;
#pragma unroll
            for (int j = 0; j < NV; ++j, next_slab<NT>(off)) {
                asm volatile("" : "+v"(keep[j]));
                if (put && has(j)) {
                    float v[N];
                    gradients<L>(v, keep[j], coef, B, p.c);
                    store_at(body, off, v);
                }
                if (LOOP && j < AHEAD) keep[j] = slab(next_row.body, j, off, nx.what == kScore);
            }
            if (DEEP && put) {
                for (int i = tid + NT * held; i < NT * lower; i += NT) {
                    float v[N];
                    gradients<L>(v, more[i - NT * held], coef, B, p.c);
                    store_at(body, (uint32_t)i * 16, v);
                }
            }
            if (put) put_pieces<L, NT>(body, row, tid + NT * lower, coef, B, p.c);
            if (far) put_far<L, NT>(body, row, coef, a.m, p.c);
        }
        if (!GRAD) return;
        __syncthreads();   // the listed entries over what the pass above wrote there
        if (mine >= 0) Piece<L>::put(out + mine, sh.patch[tid]);
        if (!LOOP || next >= p.T) return;
        t = next;
        row = next_row;
        x = nx;
    }
}

// ---- few rows: several workgroups each ----------------------------------------------
constexpr int kPartThreads = 256;
constexpr int kSplitRows = 96;                  // more rows than this go one workgroup each
constexpr int64_t kSplitGrad = 192 << 10, kSplitSum = 400 << 10;     // ... and shorter ones (bytes)
struct SplitParams {
    Part *part;                     // [T][S]
    float *z;                       // [T][k] the listed logits
    int S, seg;                     // segments of a row, elements of each (the last one's may be fewer)
};

template <typename L> __global__ __launch_bounds__(kPartThreads) void k_opd_part(LossParams<L> p, SplitParams q) {
    constexpr int NT = kPartThreads;
    extern __shared__ uint32_t bits[];
    __shared__ LossShared sh;
    __shared__ Reduce<NT> red;
    const int t = blockIdx.x / q.S, seg = blockIdx.x % q.S, tid = threadIdx.x;
    const int lo = seg * q.seg, len = min(q.seg, p.V - lo);
    const Position x = read_position(p, t);
    if (x.what != kScore) return;
    const Span<const L> row(p.z + (int64_t)t * p.ld + lo, len);
    int id;
    float tq;
    read_entry(p, tid, x, id, tq);
    clear_bits<NT>(bits, bitmap_words<L>(len), sh);
    __syncthreads();
    mark_entry(id, tq, p.k, p.V, lo, row, sh, bits);
    __syncthreads();
    if (id >= lo && id < lo + len) q.z[(int64_t)t * p.k + tid] = Piece<L>::one(row.body + (id - lo - row.head));
    MaxSum<double> own{-INFINITY, 0.};
    each_piece<NT, 4, true>(row, tid, [&](u32x4 w, int i) { add_piece<L>(own, w, i, bits, p.c); });
    RowSum a = block_merge<NT>(own, p.c, red);
    if (is_far(a.m, p.c)) a.s = sum_far<L, NT>(row, bits, a.m, p.c, red.sum[1]);
    if (tid == 0) q.part[(int64_t)t * q.S + seg] = Part{a.m, a.B, a.s, sh.bad, 0};
}

template <typename L, bool GRAD>
__global__ __launch_bounds__(kPartThreads) void k_opd_apply(LossParams<L> p, SplitParams q) {
    constexpr int NT = kPartThreads;
    __shared__ LossShared sh;
    const int S = GRAD ? q.S : 1;   // workgroups of a row
    const int t = blockIdx.x / S, seg = blockIdx.x % S, tid = threadIdx.x;
    const int lo = GRAD ? seg * q.seg : 0, len = GRAD ? min(q.seg, p.V - lo) : 0;
    L *out = GRAD ? p.grad + (int64_t)t * p.ldg + lo : nullptr;
    const Position x = read_position(p, t);
    int what = x.what, id = -1;
    RowSum a{-INFINITY, 0.f, 0.};
    if (what == kScore) {
        bool bad;
        a = join_parts(q.part + (int64_t)t * q.S, q.S, p.c, bad);
        if (bad) what = kFlag;
    }
    if (what != kScore) {
        const float v = what == kSkip ? 0.f : __builtin_nanf("");
        if (seg == 0) put_constant(p, t, v);
        if (GRAD) fill_row<L, NT>(out, len, v);
        return;
    }
    float tq;
    read_entry(p, tid, x, id, tq);
    if (tid < p.k) {
        sh.id[tid] = id;
        sh.q[tid] = tq;
        sh.z[tid] = id >= 0 ? q.z[(int64_t)t * p.k + tid] : 0.f;
    }
    __syncthreads();
    finish_row(p, t, x, a, sh, seg == 0);
    if (!GRAD) return;
    const Span<const L> row(p.z + (int64_t)t * p.ld + lo, len);
    if (is_far(a.m, p.c)) put_far<L, NT>(out + row.head, row, sh.coef, a.m, p.c);
    else put_pieces<L, NT>(out + row.head, row, tid, sh.coef, sh.B, p.c);
    __syncthreads();
    if (id >= lo && id < lo + len) Piece<L>::put(out + (id - lo), sh.patch[tid]);
}

// Segments of each row: about two workgroups a compute unit in all, at least
// 4096 elements each.  The second launch takes 4 us of the host's time, so a row
// is split only where one workgroup would take longer than that over it: with
// the gradient (bf16, us for split / whole) 8 x 65536 16.8 / 14.7, 8 x 151936
// 17.2 / 28.2, 64 x 151936 17.9 / 30.1, 128 x 151936 29.9 / 30.3; without it 8 x
// 151936 bf16 15.1 / 15.9, fp32 15.0 / 17.7.
static void split_of(int T, int V, int es, bool grad, int &S, int &seg) {
    S = 512 / (T > 0 ? T : 1);
    if (S > kMaxParts) S = kMaxParts;
    if (S > V / 4096) S = V / 4096;
    if (S < 2 || T > kSplitRows || (int64_t)V * es < (grad ? kSplitGrad : kSplitSum)) { S = 1; seg = V; return; }
    seg = ((V + S - 1) / S + 255) / 256 * 256;
    S = (V + seg - 1) / seg;
}
int64_t opd_loss_work_bytes(int T, int V, int k, int es, bool grad) {
    int S, seg;
    split_of(T, V, es, grad, S, seg);
    return S > 1 ? (int64_t)T * S * (int64_t)sizeof(Part) + (int64_t)T * k * 4 : 0;
}

// Workgroups of a launch: one a row, or where a workgroup fills a compute unit
// (its registers hold a long row) one a compute unit, which takes several rows.
static int compute_units() {
    int dev = 0, n = 0;
    if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess) return 256;
    return n;
}
template <typename L, int NT, int NV, int STEP, bool GRAD> static int launch_rows(LossParams<L> p, hipStream_t s) {
    size_t lds = (size_t)bitmap_words<L>(p.V) * 4;
    int grid = p.T;
    if (kTakesSeveral<NT, NV>) {
        const int cus = compute_units();
        if (grid > cus) grid = cus;
    }
    if (kSpills<NT, NV>) {
        // beside the bitmap and the entries, a compute unit's 160 KB (for one workgroup of 512 or two of 256) hold more slabs
        const int left = p.pieces / NT - NV;
        const int room = (int)((kLdsBytes / (NT == 512 ? 1 : 2) - sizeof(LossShared) - 1024 - lds) / (NT * 16));
        p.spill = left < 0 ? 0 : left < room ? left : room;
        lds += (size_t)p.spill * NT * 16;
    }
    return launch(k_opd_loss<L, NT, NV, STEP, GRAD>, grid, NT, lds, s, p) ? PIPO_OK : PIPO_EHIP;
}

template <typename L> static int launch_split(const LossParams<L> &p, SplitParams q, hipStream_t s) {
    bool ok = launch(k_opd_part<L>, p.T * q.S, kPartThreads, (size_t)bitmap_words<L>(q.seg) * 4, s, p, q);
    if (p.grad) ok = ok && launch(k_opd_apply<L, true>, p.T * q.S, kPartThreads, 0, s, p, q);
    else ok = ok && launch(k_opd_apply<L, false>, p.T, kPartThreads, 0, s, p, q);
    return ok ? PIPO_OK : PIPO_EHIP;
}

template <typename L> static int launch_loss(LossParams<L> p, void *work, hipStream_t s) {
    if (work && opd_loss_work_bytes(p.T, p.V, p.k, sizeof(L), p.grad != nullptr) > 0) {
        SplitParams q;
        split_of(p.T, p.V, sizeof(L), p.grad != nullptr, q.S, q.seg);
        q.part = (Part *)work;
        q.z = (float *)(q.part + (int64_t)p.T * q.S);
        return launch_split(p, q, s);
    }
    const int n = p.pieces = least_whole(p.z, p.ld, p.T, p.V);
    if (!p.grad) {
        // Few rows: all of a compute unit's waves on each; many short ones: several rows to a compute unit.  Four / eight /
        // sixteen waves, logits from memory, us: 128 x 151936 fp32 36 / 24 / 20, 256 x 32003 bf16 11.7 / 10.6 / 9.7,
        // 512 x 32003 bf16 14.1 / 13.2 / 13.5, 2048 x 8192 bf16 14 / 16 / 24, 2048 x 32003 bf16 30 / 37 / 43,
        // 2048 x 151936 bf16 109 / 103 / 104.
        if (p.T <= 256 && n >= 4000) return launch_rows<L, 1024, 4, 4, false>(p, s);
        if (p.T > 1024 && n <= 256 * 32) return launch_rows<L, 256, 4, 4, false>(p, s);
        return launch_rows<L, 512, 4, 4, false>(p, s);
    }
    // Workgroups of four waves, as many to a compute unit as their registers allow (two with 44 slabs): while one sums
    // or finishes a row, others load and write.  Only rows of which two leave most to be read again go to one workgroup
    // of eight waves a compute unit, which holds twice as much.  With the gradient, two of four waves / one of eight,
    // logits from memory, in us: bf16 2048 x 151936 248 / 253, 2048 x 168000 279 / 281, 1187 x 262144 272 / 263; fp32
    // 1944 x 80000 247 / 248, 2048 x 100000 327 / 312, 2048 x 151936 525 / 512: the same up to some 80 slabs.
    if (n < 256 * 3) return launch_rows<L, 256, 2, 2, true>(p, s);
    if (n < 256 * 5) return launch_rows<L, 256, 4, 2, true>(p, s);
    if (n < 256 * 7) return launch_rows<L, 256, 6, 2, true>(p, s);
    if (n < 256 * 9) return launch_rows<L, 256, 8, 2, true>(p, s);
    if (n < 256 * 13) return launch_rows<L, 256, 12, 4, true>(p, s);
    if (n < 256 * 17) return launch_rows<L, 256, 16, 4, true>(p, s);
    if (n < 256 * 21) return launch_rows<L, 256, 20, 4, true>(p, s);
    if (n < 256 * 26) return launch_rows<L, 256, 24, 4, true>(p, s);
    if (n < 256 * 30) return launch_rows<L, 256, 29, 4, true>(p, s);
    if (n < 256 * 35) return launch_rows<L, 256, 34, 5, true>(p, s);
    if (n < 256 * 40) return launch_rows<L, 256, 39, 5, true>(p, s);
    if (n < 256 * 82) return launch_rows<L, 256, 44, 5, true>(p, s);
    return launch_rows<L, 512, sizeof(L) == 4 ? 32 : 34, 4, true>(p, s);    // (slabs that fit beside the other values)
}

// ---- checks ---------------------------------------------------------------------
static bool aligned(const void *p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
// Rows of V elements at stride ld (elements of es bytes) starting at a and at
// b, T of each: the same rows, or no element in common.
bool same_or_apart(const void *a, int64_t lda, const void *b, int64_t ldb, int64_t T, int64_t V, int64_t es) {
    const int64_t x = (int64_t)(uintptr_t)a, y = (int64_t)(uintptr_t)b;
    if (x == y && (lda == ldb || T == 1)) return true;
    if (x + ((T - 1) * lda + V) * es <= y || y + ((T - 1) * ldb + V) * es <= x) return true;
    if (lda != ldb || T == 1) return false;
    int64_t off = (y - x) % (lda * es);     // rows of one buffer side by side
    if (off < 0) off += lda * es;
    return off >= V * es && off <= (lda - V) * es;
}

bool opd_rows_ok(int32_t T, int32_t V, const void *z, int64_t ld, double temperature, size_t es) {
    return T >= 0 && T <= kOpdMaxRows && V >= 1 && V <= kOpdMaxVocab && (T <= 1 || (ld >= V && ld <= kOpdMaxStride)) && (T == 0 || (z && aligned(z, es))) &&
           temperature >= 1e-5 && temperature <= 1e5;
}

bool opd_work_ok(const void *work, int64_t work_bytes, int64_t need) {
    return !work || (aligned(work, 16) && work_bytes >= need);
}

template <typename L>
static int check_common(const LossParams<L> &p, double temperature, const void *work, int64_t work_bytes) {
    if (!opd_rows_ok(p.T, p.V, p.z, p.ld, temperature, sizeof(L))) return PIPO_EINVAL;
    if (p.T == 0) return PIPO_OK;
    if (!p.loss) return PIPO_EINVAL;
    if (p.grad && (!aligned(p.grad, sizeof(L)) || (p.T > 1 && (p.ldg < p.V || p.ldg > kOpdMaxStride)) ||
                   !same_or_apart(p.z, p.ld, p.grad, p.ldg, p.T, p.V, sizeof(L))))
        return PIPO_EINVAL;
    return opd_work_ok(work, work_bytes, opd_loss_work_bytes(p.T, p.V, p.k, sizeof(L), p.grad != nullptr)) ? PIPO_OK : PIPO_EINVAL;
}

template <typename L>
static int distill(int32_t T, int32_t V, const L *d_logits, int64_t ld, int32_t Tt, int32_t k, const int32_t *d_ids,
                   const float *d_logp, const float *d_tail, const int32_t *d_teacher_rows, const int32_t *d_labels,
                   int32_t kind, double beta, double temperature, const float *d_scale, float *d_loss, L *d_grad,
                   int64_t ld_grad, void *d_work, int64_t work_bytes, void *stream) {
    LossParams<L> p{};
    p.z = d_logits; p.ld = ld; p.T = T; p.V = V; p.kind = kind; p.beta = beta;
    p.Tt = Tt; p.k = k; p.ids = d_ids; p.q = d_logp; p.q_rest = d_tail; p.rows = d_teacher_rows;
    p.labels = d_labels; p.scale = d_scale; p.loss = d_loss; p.grad = d_grad; p.ldg = ld_grad;
    const int rc = check_common(p, temperature, d_work, work_bytes);
    if (rc != PIPO_OK) return rc;
    if (Tt < (T > 0 ? 1 : 0) || k < 1 || k > kEntries || kind < PIPO_OPD_FORWARD || kind > PIPO_OPD_JSD) return PIPO_EINVAL;
    if (kind == PIPO_OPD_JSD && !(beta > 0. && beta < 1.)) return PIPO_EINVAL;
    if (T == 0) return PIPO_OK;
    if (!d_ids || !d_logp) return PIPO_EINVAL;
    p.c = exp_scale(temperature);
    return launch_loss(p, d_work, (hipStream_t)stream);
}

template <typename L>
static int policy(int32_t T, int32_t V, const L *d_logits, int64_t ld, const int32_t *d_labels, const float *d_adv,
                  const float *d_old_logp, const float *d_ref_logp, double clip_low, double clip_high, double kl_coef,
                  double temperature, const float *d_scale, float *d_loss, float *d_logp, float *d_kl, L *d_grad,
                  int64_t ld_grad, void *d_work, int64_t work_bytes, void *stream) {
    LossParams<L> p{};
    p.z = d_logits; p.ld = ld; p.T = T; p.V = V; p.kind = kPolicy; p.k = 1;
    p.adv = d_adv; p.old_lp = d_old_logp; p.ref_lp = d_ref_logp;
    p.clip_lo = clip_low; p.clip_hi = clip_high; p.kl_coef = kl_coef;
    p.labels = d_labels; p.scale = d_scale; p.loss = d_loss; p.logp = d_logp; p.kl = d_kl; p.grad = d_grad; p.ldg = ld_grad;
    const int rc = check_common(p, temperature, d_work, work_bytes);
    if (rc != PIPO_OK) return rc;
    if (!(clip_low >= 0. && clip_low <= 1.) || !(clip_high >= 0.) || !isfinite(clip_high) || !isfinite(kl_coef)) return PIPO_EINVAL;
    if (!d_ref_logp && (kl_coef != 0. || d_kl)) return PIPO_EINVAL;
    if (T == 0) return PIPO_OK;
    if (!d_labels || !d_adv) return PIPO_EINVAL;
    p.c = exp_scale(temperature);
    return launch_loss(p, d_work, (hipStream_t)stream);
}

}  // namespace pipo

using namespace pipo;

extern "C" int pipo_opd_distill(int32_t T, int32_t V, const float *d_logits, int64_t ld, int32_t Tt, int32_t k,
                                const int32_t *d_ids, const float *d_logp, const float *d_tail,
                                const int32_t *d_teacher_rows, const int32_t *d_labels, int32_t kind, double beta,
                                double temperature, const float *d_scale, float *d_loss, float *d_grad,
                                int64_t ld_grad, void *d_work, int64_t work_bytes, void *stream) {
    return distill<float>(T, V, d_logits, ld, Tt, k, d_ids, d_logp, d_tail, d_teacher_rows, d_labels, kind, beta,
                          temperature, d_scale, d_loss, d_grad, ld_grad, d_work, work_bytes, stream);
}

extern "C" int pipo_opd_distill_bf16(int32_t T, int32_t V, const uint16_t *d_logits, int64_t ld, int32_t Tt, int32_t k,
                                     const int32_t *d_ids, const float *d_logp, const float *d_tail,
                                     const int32_t *d_teacher_rows, const int32_t *d_labels, int32_t kind, double beta,
                                     double temperature, const float *d_scale, float *d_loss, uint16_t *d_grad,
                                     int64_t ld_grad, void *d_work, int64_t work_bytes, void *stream) {
    return distill<uint16_t>(T, V, d_logits, ld, Tt, k, d_ids, d_logp, d_tail, d_teacher_rows, d_labels, kind, beta,
                             temperature, d_scale, d_loss, d_grad, ld_grad, d_work, work_bytes, stream);
}

extern "C" int pipo_opd_policy(int32_t T, int32_t V, const float *d_logits, int64_t ld, const int32_t *d_labels,
                               const float *d_adv, const float *d_old_logp, const float *d_ref_logp, double clip_low,
                               double clip_high, double kl_coef, double temperature, const float *d_scale,
                               float *d_loss, float *d_logp, float *d_kl, float *d_grad, int64_t ld_grad, void *d_work,
                               int64_t work_bytes, void *stream) {
    return policy<float>(T, V, d_logits, ld, d_labels, d_adv, d_old_logp, d_ref_logp, clip_low, clip_high, kl_coef,
                         temperature, d_scale, d_loss, d_logp, d_kl, d_grad, ld_grad, d_work, work_bytes, stream);
}

extern "C" int pipo_opd_policy_bf16(int32_t T, int32_t V, const uint16_t *d_logits, int64_t ld,
                                    const int32_t *d_labels, const float *d_adv, const float *d_old_logp,
                                    const float *d_ref_logp, double clip_low, double clip_high, double kl_coef,
                                    double temperature, const float *d_scale, float *d_loss, float *d_logp,
                                    float *d_kl, uint16_t *d_grad, int64_t ld_grad, void *d_work, int64_t work_bytes,
                                    void *stream) {
    return policy<uint16_t>(T, V, d_logits, ld, d_labels, d_adv, d_old_logp, d_ref_logp, clip_low, clip_high, kl_coef,
                            temperature, d_scale, d_loss, d_logp, d_kl, d_grad, ld_grad, d_work, work_bytes, stream);
}
