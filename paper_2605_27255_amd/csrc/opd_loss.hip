// OPD losses with their gradients (App. C): the divergence of a student row
// from a teacher's top logits, and the clipped policy loss of a row's label.
//
// With x = z / temperature, both are functions of the log-probabilities of a
// few listed entries of the row (the teacher's ids; the label) and of the mass
// of all others.  For a = p df/dp of each entry and of the rest r, A = sum a:
//   dL/dz_v = (a_v - p_v A) / temperature                       v listed
//   dL/dz_v = (a_r softmax_rest(v) - p_v A) / temperature        v not listed
// so the row's gradient away from the list is exp((z_v - m) / temperature)
// times one number.  One pass over the row gives the maximum m and the sum of
// exponentials of the unlisted values (a bitmap of the listed ids in LDS drops
// them from the sum, so the rest's mass carries no cancellation even where it
// is tiny); everything per entry is 64-bit arithmetic on a handful of numbers;
// a second pass writes the gradient, and the listed entries are written over it.
// HBM-bound: V logits read, V gradients written.
//
// Where there are too few rows for the chip, each is split over several
// workgroups: k_opd_part sums a segment and gathers the listed logits,
// k_opd_apply joins the segments' sums (every workgroup for itself, from a few
// numbers) and writes its segment's gradient.
#include "opd_rows.h"
#include "pipo.h"

namespace pipo {

constexpr int kEntries = 256;       // listed entries of a row
constexpr int64_t kOpdMaxStride = (int64_t)1 << 31;   // with T < 2^31, byte offsets stay far inside 64 bits

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
};
constexpr int kPolicy = 3;

struct LossShared {
    int id[kEntries];               // listed ids, -1: an empty slot
    float z[kEntries];              // their logits
    double a[kEntries], p[kEntries];   // their a = p df/dp, and p
    float patch[kEntries];          // their gradients
    float coef;                     // the others' gradient over exp((z - m) / temperature)
    int bad;
};

// What happens at position t: not scored, flagged (no such row, label or id), or scored with k entries.
enum { kSkip, kFlag, kScore };

// What happens at position t (the same for the whole workgroup), and its teacher row.
template <typename L> __device__ __forceinline__ int position_state(const LossParams<L> &p, int t, int &y, int &trow) {
    y = p.labels ? p.labels[t] : 0;
    trow = p.rows ? p.rows[t] : t;
    if (y < 0) return kSkip;
    return (p.kind == kPolicy ? y >= p.V : (trow < 0 || trow >= p.Tt)) ? kFlag : kScore;
}
template <typename L> __device__ __forceinline__ int entry_id(const LossParams<L> &p, int j, int y, int trow) {
    if (j >= p.k) return -1;
    return p.kind == kPolicy ? y : p.ids[(int64_t)trow * p.k + j];
}
// Marks the listed ids of [lo, lo + len) in the bitmap (bit id - lo) and keeps
// all of them in LDS; sh.bad is set where one is out of range, or twice in this
// range.  Thread j brings entry j.  Ends with a barrier.
template <int NT>
__device__ __forceinline__ void mark_entries(int id, int k, int V, int lo, int len, LossShared &sh, uint32_t *bits) {
    const int tid = threadIdx.x;
    for (int i = tid; i < (len + 31) / 32; i += NT) bits[i] = 0;
    if (tid == 0) sh.bad = 0;
    __syncthreads();
    if (tid < k) {
        sh.id[tid] = id;
        const int at = id - lo;
        if (id >= V || (id >= lo && at < len && (atomicOr(&bits[at >> 5], 1u << (at & 31)) >> (at & 31) & 1u))) sh.bad = 1;
    }
    __syncthreads();
}

// The bitmap's bits of piece i (bit e: its element e is listed).
template <int N> __device__ __forceinline__ uint32_t listed_bits(const uint32_t *bits, int i) {
    const uint32_t b = ((const uint8_t *)bits)[i * N >> 3];
    return N == 8 ? b : (b >> ((i & 1) * 4)) & 15u;
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
__device__ __forceinline__ void finish_row(const LossParams<L> &p, int t, int trow, MaxSum rest, LossShared &sh,
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
        // log of the rest's unit (its sum counts multiples of it) over exp(m / temperature)
        const double unit = is_far(rest.m) ? ((double)rest.m - m) * inv : (double)ref_of(rest.m, p.c) * kLn2 - m * inv;
        const double rest_at = rest.m == -INFINITY ? 1. : exp(unit);
        sum += (double)rest.s * rest_at;     // without a rest its sum is 0 (or NaN)
        // of x - m / temperature; a row without any mass has none
        const double lse = m == -INFINITY ? (double)__builtin_nanf("") : log(sum);
        const double g = (p.scale ? (double)p.scale[t] : 1.) * inv;
        double A = 0., a_rest = 0.;
        if (p.kind == kPolicy) {
            const double lp = ((double)sh.z[0] - m) * inv - lse, py = exp(lp), adv = p.adv[t];
            const double r = p.old_lp ? exp(lp - (double)p.old_lp[t]) : exp(lp - lp);
            const double cut = fmin(fmax(r, 1. - p.clip_lo), 1. + p.clip_hi);
            const bool inside = adv * r <= adv * cut;
            double loss = -(inside ? adv * r : adv * cut), d = inside ? -adv * r : 0., kl = 0.;
            if (r != r || adv != adv) loss = d = r + adv;
            if (p.ref_lp) {
                const double far = (double)p.ref_lp[t] - lp;
                kl = expm1(far) - far;
                if (p.kl_coef != 0.) {
                    loss += p.kl_coef * kl;
                    d -= p.kl_coef * expm1(far);
                }
            }
            A = d;
            if (lane == 0) sh.patch[0] = (float)(g * (d - py * d));
            if (lane == 0 && first) {
                p.loss[t] = (float)loss;
                if (p.logp) p.logp[t] = (float)lp;
                if (p.kl) p.kl[t] = (float)kl;
            }
        } else {
            double f = 0.;
            const float *q = p.q + (int64_t)trow * p.k;
            // entry k stands for the tokens outside the list
            for (int j = lane; j < p.k + (p.q_rest ? 1 : 0); j += 64) {
                const bool out = j == p.k;
                if (!out && sh.id[j] < 0) continue;
                double lp = out ? unit + log((double)rest.s) - lse : ((double)sh.z[j] - m) * inv - lse;
                if (out && rest.s == 0.f) lp = lse == lse ? -INFINITY : lse;
                double fj, aj;
                divergence(p.kind, p.beta, lp, out ? (double)p.q_rest[trow] : (double)q[j], fj, aj);
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
            for (int j = lane; j < p.k; j += 64)
                if (sh.id[j] >= 0) sh.patch[j] = (float)(g * (sh.a[j] - sh.p[j] * A));
        }
        if (lane == 0) {
            // with no mass outside the list there is nothing to spread there
            const double k = lse != lse ? lse : rest.s == 0.f ? 0. : g * (a_rest / (double)rest.s - A * rest_at * exp(-lse));
            sh.coef = (float)k;
        }
    }
    __syncthreads();
}

template <typename L, int NT>
__device__ __forceinline__ void fill_row(L *row, int V, float v) {
    float x[Piece<L>::N];
#pragma unroll
    for (int e = 0; e < Piece<L>::N; ++e) x[e] = v;
    const int whole = V / Piece<L>::N;
    for (int i = threadIdx.x; i < whole; i += NT) store_piece(row, i, x);
    if ((int)threadIdx.x == whole % NT) store_last(row, whole, V, x);
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
__device__ __forceinline__ void add_piece(MaxSum &a, u32x4 w, int i, const uint32_t *bits, ExpScale c) {
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
__device__ __forceinline__ float sum_far(const L *row, int len, const uint32_t *bits, float m, ExpScale c, float *s_w) {
    constexpr int N = Piece<L>::N;
    float s = 0.f;
    each_piece<NT, 1>(row, (int)threadIdx.x, len, [&](u32x4 w, int i) {
        const uint32_t b = listed_bits<N>(bits, i);
#pragma unroll
        for (int e = 0; e < N; ++e) if (!(b >> e & 1u)) s += exp_diff(Piece<L>::get(w, e), m, c);
    });
    return (float)block_sum<NT>(s, s_w);
}
// A piece's gradients away from the list; those of listed elements are written over them later.
template <typename L>
__device__ __forceinline__ void put_piece(L *out, u32x4 w, int i, int len, float coef, MaxSum rest, ExpScale c) {
    constexpr int N = Piece<L>::N;
    const float B = ref_of(rest.m, c);
    float v[N];
    // c's second float matters to sums only: here it is less than one rounding of each exponent
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = coef * __builtin_amdgcn_exp2f(fmaf(Piece<L>::get(w, e), c.hi, -B));
    if ((i + 1) * N <= len) store_piece(out, i, v);
    else store_last(out, i, len, v);
}
template <typename L, int NT>
__device__ __forceinline__ void put_far(L *out, const L *row, int len, float coef, float m, ExpScale c) {
    constexpr int N = Piece<L>::N;
    each_piece<NT, 1>(row, (int)threadIdx.x, len, [&](u32x4 w, int i) {
        float v[N];
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = coef * exp_diff(Piece<L>::get(w, e), m, c);
        if ((i + 1) * N <= len) store_piece(out, i, v);
        else store_last(out, i, len, v);
    });
}

// One workgroup per position.  Its first NV pieces a thread stay in registers
// between the two passes; the rest of a longer row is read again.
template <typename L, int NT, int NV, bool GRAD>
__global__ __launch_bounds__(NT) void k_opd_loss(LossParams<L> p) {
    extern __shared__ uint32_t bits[];
    __shared__ LossShared sh;
    __shared__ float red[3][NT / 64];
    const int t = blockIdx.x, tid = threadIdx.x, V = p.V, whole = V / Piece<L>::N;
    const L *row = p.z + (int64_t)t * p.ld;
    int y, trow, what = position_state(p, t, y, trow);
    u32x4 keep[NV ? NV : 1];
    float zj = 0.f;
    if (what == kScore) {
        const int id = entry_id(p, tid, y, trow);
#pragma unroll
        for (int j = 0; j < NV; ++j)      // in flight while the entries are marked
            if (tid + NT * j < whole) keep[j] = load_piece(row, tid + NT * j);
        mark_entries<NT>(id, p.k, V, 0, V, sh, bits);
        if (sh.bad) what = kFlag;
        else if (id >= 0) zj = Piece<L>::one(row + id);
    }
    if (what != kScore) {
        const float v = what == kSkip ? 0.f : __builtin_nanf("");
        put_constant(p, t, v);
        if (GRAD) fill_row<L, NT>(p.grad + (int64_t)t * p.ldg, V, v);
        return;
    }
    MaxSum a{-INFINITY, 0.f};
#pragma unroll
    for (int j = 0; j < NV; ++j)
        if (tid + NT * j < whole) add_piece<L>(a, keep[j], tid + NT * j, bits, p.c);
    each_piece<NT, 4>(row, tid + NT * NV, V, [&](u32x4 w, int i) { add_piece<L>(a, w, i, bits, p.c); });
    if (tid < p.k) sh.z[tid] = zj;
    a = block_merge<NT>(a, p.c, red);
    const bool far = is_far(a.m);
    if (far) a.s = sum_far<L, NT>(row, V, bits, a.m, p.c, red[2]);
    finish_row(p, t, trow, a, sh);
    if (!GRAD) return;
    L *out = p.grad + (int64_t)t * p.ldg;
    const float coef = sh.coef;
    if (far) {
        put_far<L, NT>(out, row, V, coef, a.m, p.c);
    } else {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            asm volatile("" : "+v"(keep[j]));   // unpacked again: the first pass' floats would take twice the registers
            if (tid + NT * j < whole) put_piece(out, keep[j], tid + NT * j, V, coef, a, p.c);
        }
        each_piece<NT, 4>(row, tid + NT * NV, V, [&](u32x4 w, int i) { put_piece(out, w, i, V, coef, a, p.c); });
    }
    __syncthreads();   // the listed entries over what the pass above wrote there
    if (tid < p.k && sh.id[tid] >= 0) Piece<L>::put(out + sh.id[tid], sh.patch[tid]);
}

// ---- few rows: several workgroups each ----------------------------------------------
constexpr int kPartThreads = 256;
constexpr int kSplitRows = 160;     // more rows than this go one workgroup each
struct SplitParams {
    Part *part;                     // [T][S]
    float *z;                       // [T][k] the listed logits
    int S, seg;                     // segments of a row, elements of each (the last one's may be fewer)
};

template <typename L> __global__ __launch_bounds__(kPartThreads) void k_opd_part(LossParams<L> p, SplitParams q) {
    constexpr int NT = kPartThreads;
    extern __shared__ uint32_t bits[];
    __shared__ LossShared sh;
    __shared__ float red[3][NT / 64];
    const int t = blockIdx.x / q.S, seg = blockIdx.x % q.S, tid = threadIdx.x;
    const int lo = seg * q.seg, len = min(q.seg, p.V - lo);
    int y, trow;
    if (position_state(p, t, y, trow) != kScore) return;
    const L *row = p.z + (int64_t)t * p.ld + lo;
    const int id = entry_id(p, tid, y, trow);
    mark_entries<NT>(id, p.k, p.V, lo, len, sh, bits);
    if (id >= lo && id < lo + len) q.z[(int64_t)t * p.k + tid] = Piece<L>::one(row + (id - lo));
    MaxSum a{-INFINITY, 0.f};
    each_piece<NT, 4>(row, tid, len, [&](u32x4 w, int i) { add_piece<L>(a, w, i, bits, p.c); });
    a = block_merge<NT>(a, p.c, red);
    if (is_far(a.m)) a.s = sum_far<L, NT>(row, len, bits, a.m, p.c, red[2]);
    if (tid == 0) q.part[(int64_t)t * q.S + seg] = Part{a.m, a.s, sh.bad, 0};
}

template <typename L, bool GRAD>
__global__ __launch_bounds__(kPartThreads) void k_opd_apply(LossParams<L> p, SplitParams q) {
    constexpr int NT = kPartThreads;
    __shared__ LossShared sh;
    const int S = GRAD ? q.S : 1;   // workgroups of a row
    const int t = blockIdx.x / S, seg = blockIdx.x % S, tid = threadIdx.x;
    const int lo = GRAD ? seg * q.seg : 0, len = GRAD ? min(q.seg, p.V - lo) : 0;
    L *out = GRAD ? p.grad + (int64_t)t * p.ldg + lo : nullptr;
    int y, trow, what = position_state(p, t, y, trow), id = -1;
    MaxSum a{-INFINITY, 0.f};
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
    if (tid < p.k) {
        id = entry_id(p, tid, y, trow);
        sh.id[tid] = id;
        sh.z[tid] = id >= 0 ? q.z[(int64_t)t * p.k + tid] : 0.f;
    }
    __syncthreads();
    finish_row(p, t, trow, a, sh, seg == 0);
    if (!GRAD) return;
    const L *row = p.z + (int64_t)t * p.ld + lo;
    const float coef = sh.coef;
    if (is_far(a.m)) put_far<L, NT>(out, row, len, coef, a.m, p.c);
    else each_piece<NT, 4>(row, tid, len, [&](u32x4 w, int i) { put_piece(out, w, i, len, coef, a, p.c); });
    __syncthreads();
    if (id >= lo && id < lo + len) Piece<L>::put(out + (id - lo), sh.patch[tid]);
}

// Segments of each row: about two workgroups a compute unit in all, at least 4096 elements each.
static void split_of(int T, int V, int &S, int &seg) {
    S = 512 / (T > 0 ? T : 1);
    if (S > kMaxParts) S = kMaxParts;
    if (S > V / 4096) S = V / 4096;
    if (S < 2 || T > kSplitRows) { S = 1; seg = V; return; }
    seg = ((V + S - 1) / S + 255) / 256 * 256;
    S = (V + seg - 1) / seg;
}
static int64_t split_bytes(int T, int V, int k) {
    int S, seg;
    split_of(T, V, S, seg);
    return S > 1 ? (int64_t)T * S * (int64_t)sizeof(Part) + (int64_t)T * k * 4 : 0;
}
int64_t opd_loss_work_bytes(int T, int V, int k) { return split_bytes(T, V, k); }

template <typename L, int NT, int NV, bool GRAD> static int launch_rows(const LossParams<L> &p, hipStream_t s) {
    const size_t lds = (size_t)((p.V + 31) / 32) * 4;
    hipLaunchKernelGGL((k_opd_loss<L, NT, NV, GRAD>), dim3(p.T), dim3(NT), lds, s, p);
    return hipGetLastError() == hipSuccess ? PIPO_OK : PIPO_EHIP;
}

template <typename L> static int launch_split(const LossParams<L> &p, SplitParams q, hipStream_t s) {
    const dim3 grid((unsigned)(p.T * q.S)), block(kPartThreads);
    hipLaunchKernelGGL(k_opd_part<L>, grid, block, (size_t)((q.seg + 31) / 32) * 4, s, p, q);
    if (p.grad) hipLaunchKernelGGL((k_opd_apply<L, true>), grid, block, 0, s, p, q);
    else hipLaunchKernelGGL((k_opd_apply<L, false>), dim3(p.T), block, 0, s, p, q);
    return hipGetLastError() == hipSuccess ? PIPO_OK : PIPO_EHIP;
}

template <typename L> static int launch_loss(const LossParams<L> &p, void *work, hipStream_t s) {
    const int n = (p.V + Piece<L>::N - 1) / Piece<L>::N;
    if (work && split_bytes(p.T, p.V, p.k) > 0) {
        SplitParams q;
        split_of(p.T, p.V, q.S, q.seg);
        q.part = (Part *)work;
        q.z = (float *)(q.part + (int64_t)p.T * q.S);
        return launch_split(p, q, s);
    }
    if (!p.grad) {
        if (n <= 256 * 32) return launch_rows<L, 256, 0, false>(p, s);
        return launch_rows<L, 512, 0, false>(p, s);
    }
    if (n <= 256 * 2) return launch_rows<L, 256, 2, true>(p, s);
    if (n <= 256 * 4) return launch_rows<L, 256, 4, true>(p, s);
    if (n <= 256 * 8) return launch_rows<L, 256, 8, true>(p, s);
    if (n <= 512 * 8) return launch_rows<L, 512, 8, true>(p, s);
    if (n <= 512 * 16) return launch_rows<L, 512, 16, true>(p, s);
    if (n <= 512 * 24) return launch_rows<L, 512, 24, true>(p, s);
    if (n <= 512 * 32) return launch_rows<L, 512, 32, true>(p, s);
    return launch_rows<L, 512, 38, true>(p, s);
}

// ---- checks ---------------------------------------------------------------------
static bool aligned(const void *p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
// Rows of V elements at stride ld (elements of es bytes) starting at a and at
// b, T of each: the same rows, or no element in common.
static bool same_or_apart(const void *a, int64_t lda, const void *b, int64_t ldb, int64_t T, int64_t V, int64_t es) {
    const int64_t x = (int64_t)(uintptr_t)a, y = (int64_t)(uintptr_t)b;
    if (x == y && (lda == ldb || T == 1)) return true;
    if (x + ((T - 1) * lda + V) * es <= y || y + ((T - 1) * ldb + V) * es <= x) return true;
    if (lda != ldb || T == 1) return false;
    int64_t off = (y - x) % (lda * es);     // rows of one buffer side by side
    if (off < 0) off += lda * es;
    return off >= V * es && off <= (lda - V) * es;
}

bool opd_rows_ok(int32_t T, int32_t V, const void *z, int64_t ld, double temperature, size_t es) {
    return T >= 0 && V >= 1 && V <= kOpdMaxVocab && (T <= 1 || (ld >= V && ld <= kOpdMaxStride)) && (T == 0 || (z && aligned(z, es))) &&
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
    return opd_work_ok(work, work_bytes, split_bytes(p.T, p.V, p.k)) ? PIPO_OK : PIPO_EINVAL;
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
    if (Tt < 1 || k < 1 || k > kEntries || kind < PIPO_OPD_FORWARD || kind > PIPO_OPD_JSD) return PIPO_EINVAL;
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
