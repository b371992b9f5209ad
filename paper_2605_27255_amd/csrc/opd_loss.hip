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
#include "opd_rows.h"
#include "pipo.h"

namespace pipo {

constexpr int kEntries = 256;       // listed entries of a row
constexpr int kOpdMaxVocab = 1 << 19;
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
    MaxSum red[16];
    int id[kEntries];               // listed ids, -1: an empty slot
    float z[kEntries];              // their logits
    float patch[kEntries];          // their gradients
    float coef;                     // the others' gradient over exp((z - m) / temperature)
    int bad;
};

// What happens at position t: not scored, flagged (no such row, label or id), or scored with k entries.
enum { kSkip, kFlag, kScore };

// Reads position t's entries into LDS and marks them in the bitmap (bit id of
// a row's ids); ends with a barrier.
template <typename L, int NT>
__device__ __forceinline__ int list_entries(const LossParams<L> &p, int t, LossShared &sh, uint32_t *bits, int &trow) {
    const int tid = threadIdx.x;
    const int y = p.labels ? p.labels[t] : 0;
    if (y < 0) return kSkip;
    trow = p.rows ? p.rows[t] : t;
    if (p.kind == kPolicy ? y >= p.V : (trow < 0 || trow >= p.Tt)) return kFlag;
    for (int i = tid; i < (p.V + 31) / 32; i += NT) bits[i] = 0;
    if (tid == 0) sh.bad = 0;
    __syncthreads();
    for (int j = tid; j < p.k; j += NT) {
        const int id = p.kind == kPolicy ? y : p.ids[(int64_t)trow * p.k + j];
        float z = 0.f;
        if (id >= p.V) sh.bad = 1;
        else if (id >= 0) {
            z = Piece<L>::one(p.z + (int64_t)t * p.ld + id);
            if (atomicOr(&bits[id >> 5], 1u << (id & 31)) >> (id & 31) & 1u) sh.bad = 1;   // listed twice
        }
        sh.id[j] = id;
        sh.z[j] = z;
    }
    __syncthreads();
    return sh.bad ? kFlag : kScore;
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
// position's outputs and its gradient's numbers; ends with a barrier.
template <typename L>
__device__ __forceinline__ void finish_row(const LossParams<L> &p, int t, int trow, MaxSum rest, LossShared &sh) {
    if (threadIdx.x < 64) {
        const int lane = threadIdx.x;
        const double inv = p.c.inv;
        double m = rest.m;
        for (int j = lane; j < p.k; j += 64) if (sh.id[j] >= 0) m = fmax(m, (double)sh.z[j]);
        for (int o = 32; o > 0; o >>= 1) m = fmax(m, __shfl_xor(m, o));
        double sum = 0.;
        for (int j = lane; j < p.k; j += 64) if (sh.id[j] >= 0) sum += exp(((double)sh.z[j] - m) * inv);
        sum = wave_sum_f64(sum);
        const double rest_ref = ref_of(rest.m);
        const double rest_at = rest.m == -INFINITY ? 0. : exp((rest_ref - m) * inv);   // exp((rest.m - m) / temperature)
        sum += (double)rest.s * (rest.m == -INFINITY ? 1. : rest_at);
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
            if (lane == 0) {
                p.loss[t] = (float)loss;
                if (p.logp) p.logp[t] = (float)lp;
                if (p.kl) p.kl[t] = (float)kl;
                sh.patch[0] = (float)(g * (d - py * d));
            }
        } else {
            double f = 0.;
            const float *q = p.q + (int64_t)trow * p.k;
            for (int j = lane; j < p.k; j += 64) {
                if (sh.id[j] < 0) continue;
                double fj, aj;
                divergence(p.kind, p.beta, ((double)sh.z[j] - m) * inv - lse, (double)q[j], fj, aj);
                f += fj;
                A += aj;
            }
            f = wave_sum_f64(f);
            A = wave_sum_f64(A);
            if (p.q_rest) {
                double fr;
                const double lp = rest.s == 0.f ? -INFINITY + lse * 0. : (rest_ref - m) * inv + log((double)rest.s) - lse;
                divergence(p.kind, p.beta, lp, (double)p.q_rest[trow], fr, a_rest);
                f += fr;
                A += a_rest;
            }
            if (!(lse == lse)) f = lse;
            if (lane == 0) p.loss[t] = (float)f;
            for (int j = lane; j < p.k; j += 64) {
                if (sh.id[j] < 0) continue;
                double fj, aj;
                const double lp = ((double)sh.z[j] - m) * inv - lse;
                divergence(p.kind, p.beta, lp, (double)q[j], fj, aj);
                sh.patch[j] = (float)(g * (aj - exp(lp) * A));
            }
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
    for (int i = threadIdx.x; i * Piece<L>::N < V; i += NT) store_piece(row, i, V, x);
}

// A position that is not scored (zeros) or flagged (NaN).
template <typename L>
__device__ __forceinline__ void put_constant(const LossParams<L> &p, int t, float v) {
    if (threadIdx.x != 0) return;
    p.loss[t] = v;
    if (p.logp) p.logp[t] = v;
    if (p.kl) p.kl[t] = v;
}

// One workgroup per position.
template <typename L, int NT, bool GRAD>
__global__ __launch_bounds__(NT) void k_opd_loss(LossParams<L> p) {
    constexpr int N = Piece<L>::N;
    extern __shared__ uint32_t bits[];
    __shared__ LossShared sh;
    const int t = blockIdx.x, tid = threadIdx.x, V = p.V, n = (V + N - 1) / N;
    const L *row = p.z + (int64_t)t * p.ld;
    int trow = 0;
    const int what = list_entries<L, NT>(p, t, sh, bits, trow);
    if (what != kScore) {
        const float v = what == kSkip ? 0.f : __builtin_nanf("");
        put_constant(p, t, v);
        if (GRAD) fill_row<L, NT>(p.grad + (int64_t)t * p.ldg, V, v);
        return;
    }
    MaxSum a{-INFINITY, 0.f};
    for (int i = tid; i < n; i += NT) {
        const u32x4 w = load_piece(row, i, V);
        const uint32_t b = listed_bits<N>(bits, i);
        float v[N];
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = Piece<L>::get(w, e);
        if (b) {
#pragma unroll
            for (int e = 0; e < N; ++e) if (b >> e & 1u) v[e] = -INFINITY;
        }
        add_values<N>(a, v, p.c);
    }
    a = block_merge<NT>(a, p.c, sh.red);
    finish_row(p, t, trow, a, sh);
    if (!GRAD) return;
    L *out = p.grad + (int64_t)t * p.ldg;
    const float coef = sh.coef, m = ref_of(a.m);
    for (int i = tid; i < n; i += NT) {
        const u32x4 w = load_piece(row, i, V);
        float v[N];
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = coef * exp_diff(Piece<L>::get(w, e), m, p.c);
        store_piece(out, i, V, v);
    }
    __syncthreads();   // the listed entries over what the pass above wrote there
    for (int j = tid; j < p.k; j += NT) if (sh.id[j] >= 0) Piece<L>::put(out + sh.id[j], sh.patch[j]);
}

template <typename L, int NT> static int launch_rows(const LossParams<L> &p, hipStream_t s) {
    const size_t lds = (size_t)((p.V + 31) / 32) * 4;
    if (p.grad) hipLaunchKernelGGL((k_opd_loss<L, NT, true>), dim3(p.T), dim3(NT), lds, s, p);
    else hipLaunchKernelGGL((k_opd_loss<L, NT, false>), dim3(p.T), dim3(NT), lds, s, p);
    return hipGetLastError() == hipSuccess ? PIPO_OK : PIPO_EHIP;
}

template <typename L> static int launch_loss(const LossParams<L> &p, void *work, int64_t work_bytes, hipStream_t s) {
    (void)work; (void)work_bytes;
    return p.V > 16384 ? launch_rows<L, 1024>(p, s) : launch_rows<L, 256>(p, s);
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
           temperature > 0. && isfinite(temperature) && isfinite(1.4426950408889634 / temperature) &&
           1.4426950408889634 / temperature < 1e30 && 1.4426950408889634 / temperature > 1e-30;
}

template <typename L> static int check_common(const LossParams<L> &p, double temperature) {
    if (!opd_rows_ok(p.T, p.V, p.z, p.ld, temperature, sizeof(L))) return PIPO_EINVAL;
    if (p.T == 0) return PIPO_OK;
    if (!p.loss) return PIPO_EINVAL;
    if (p.grad && (!aligned(p.grad, sizeof(L)) || (p.T > 1 && (p.ldg < p.V || p.ldg > kOpdMaxStride)) ||
                   !same_or_apart(p.z, p.ld, p.grad, p.ldg, p.T, p.V, sizeof(L))))
        return PIPO_EINVAL;
    return PIPO_OK;
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
    const int rc = check_common(p, temperature);
    if (rc != PIPO_OK) return rc;
    if (Tt < 1 || k < 1 || k > kEntries || kind < PIPO_OPD_FORWARD || kind > PIPO_OPD_JSD) return PIPO_EINVAL;
    if (kind == PIPO_OPD_JSD && !(beta > 0. && beta < 1.)) return PIPO_EINVAL;
    if (T == 0) return PIPO_OK;
    if (!d_ids || !d_logp) return PIPO_EINVAL;
    p.c = exp_scale(temperature);
    return launch_loss(p, d_work, work_bytes, (hipStream_t)stream);
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
    const int rc = check_common(p, temperature);
    if (rc != PIPO_OK) return rc;
    if (!(clip_low >= 0. && clip_low <= 1.) || !(clip_high >= 0.) || !isfinite(clip_high) || !isfinite(kl_coef)) return PIPO_EINVAL;
    if (!d_ref_logp && (kl_coef != 0. || d_kl)) return PIPO_EINVAL;
    if (T == 0) return PIPO_OK;
    if (!d_labels || !d_adv) return PIPO_EINVAL;
    p.c = exp_scale(temperature);
    return launch_loss(p, d_work, work_bytes, (hipStream_t)stream);
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
