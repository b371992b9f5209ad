// Verification of drafted tokens against a target's logits from given random numbers.
//
// Draft i of a request is accepted while u_i q_i < p_i; the token behind the accepted ones
// is drawn from max(p - q, 0), or p, by the inverse of its running sum over the ids.
// Three launches: each segment of each row to its maximum and its sum of exponentials of
// differences to it (every logit read once, from HBM: what bounds it); the accepted drafts
// of a request from a few numbers a row, and the masses of the segments of the one or
// two rows that the next token is drawn from (again from the caches); the segment
// that holds the drawn mass, element by element.  Exponentials are fp32 of exact
// differences, everything that a choice hangs on is added and compared in 64 bits.
#include "kv8.h"

namespace pipo {

constexpr int kSegThreads = 256, kSegEach = 32, kSeg = kSegThreads * kSegEach;  // logits of a segment
static_assert((int64_t)kSeg * kMaxParts >= kOpdMaxVocab, "a lane for each segment of a row");

struct SegPart { double s; float m; int32_t id; };      // sum of exp(x - m), the maximum, its lowest id
struct Verdict { double p_inv, q_inv; float p_m, q_m; int32_t kind, row; };     // what the next token is drawn from
enum { kFromP = 0, kFromRest = 1, kWithout = 2, kNone = 3, kToken = 4 };        // p; max(p - q, 0); p without the draft; nothing; a known one

template <typename L> struct VerifyParams {
    const L *z; int64_t ld;
    const L *d; int64_t ld_request, ld_draft;   // the drafter's (NULL: none)
    const int32_t *starts, *drafts;
    const float *u;
    int R, K, V, rows, S, greedy;
    ExpScale c;
    int32_t *tokens, *accepted;
    SegPart *part;                  // [target rows R (K + 1), then drafter rows R K][S]
    double *mass;                   // [R][S]
    Verdict *verdict;               // [R]
};

// Rows of request r: the first, and the number of drafts that have one (-1: no rows at all).
template <typename L> __device__ __forceinline__ int rows_of(const VerifyParams<L> &p, int r, int &first) {
    int n = p.K + 1;
    first = r * (p.K + 1);
    if (p.starts) {
        first = max(p.starts[r], 0);
        n = min(p.starts[r + 1], p.rows) - first;
    } else {
        n = min(n, p.rows - first);
    }
    n = min(n - 1, p.K);
    if (n < 0) return -1;
    // (up to 63 drafts: a lane each)
    const int lane = threadIdx.x & 63;
    const uint64_t ends = __ballot(lane >= n || p.drafts[(int64_t)r * p.K + lane] < 0);
    return __builtin_ctzll(ends);
}
// Logits [seg kSeg, ...) of a row, kSegEach a thread: thread t's are pieces t, t + kSegThreads, ...
template <typename L, typename F> __device__ __forceinline__ void each_of(const L *row, int lo, int n, F f) {
    constexpr int N = Piece<L>::N, P = kSegEach / N;
    u32x4 w[P];
    const L *at = row + lo;
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const int e0 = ((int)threadIdx.x + i * kSegThreads) * N;
        if (e0 + N <= n) w[i] = *(const typename Piece<L>::raw_t *)(at + e0);
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const int e0 = ((int)threadIdx.x + i * kSegThreads) * N;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            float v = -INFINITY;
            if (e0 + N <= n) v = Piece<L>::get(w[i], e);
            else if (e0 + e < n) v = Piece<L>::one(at + e0 + e);
            f(v, lo + e0 + e, i * N + e);
        }
    }
}

template <typename L> __global__ __launch_bounds__(kSegThreads) void k_verify_rows(VerifyParams<L> p) {
    const int seg = blockIdx.x % p.S, line = blockIdx.x / p.S, targets = p.R * (p.K + 1);
    const L *row;
    int first, r, n;
    if (line < targets) {
        r = line / (p.K + 1);
        const int i = line - r * (p.K + 1);
        n = rows_of(p, r, first);
        if (i > n) return;
        row = p.z + (first + i) * p.ld;
    } else {
        r = (line - targets) / p.K;
        const int i = line - targets - r * p.K;
        n = rows_of(p, r, first);
        if (i >= n) return;
        row = p.d + r * p.ld_request + i * p.ld_draft;
    }
    __shared__ float s_m[kSegThreads / 64];
    __shared__ double s_s[kSegThreads / 64];
    __shared__ int s_id[kSegThreads / 64];
    const int lo = seg * kSeg, len = min(kSeg, p.V - lo);
    float v[kSegEach], m = -INFINITY;
    each_of(row, lo, len, [&](float x, int, int k) { v[k] = x; m = fmaxf(m, x); });
    m = block_max<kSegThreads>(m, s_m);
    float sum = 0.f;
    if (m != -INFINITY) {
#pragma unroll
        for (int k = 0; k < kSegEach; ++k) sum += exp_diff(v[k], m, p.c);
    } else {
#pragma unroll
        for (int k = 0; k < kSegEach; ++k) sum += v[k] != v[k] ? v[k] : 0.f;
    }
    const double s = block_sum<kSegThreads>((double)sum, s_s);
    int id = p.V;
    if (p.greedy) {
        constexpr int N = Piece<L>::N;
#pragma unroll
        for (int k = kSegEach - 1; k >= 0; --k)
            if (v[k] == m) id = lo + ((int)threadIdx.x + k / N * kSegThreads) * N + k % N;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) id = min(id, __shfl_xor(id, o));
        if ((threadIdx.x & 63) == 0) s_id[threadIdx.x >> 6] = id;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kSegThreads / 64; ++w) id = min(id, s_id[w]);
    }
    if (threadIdx.x == 0) p.part[(int64_t)line * p.S + seg] = SegPart{s, m, id};
}

// A row from its segments, in every lane of a wave: maximum, 1 / sum (0: the row is bad), its largest logit's id.
struct RowStat { float m; double inv; int id; };
__device__ __forceinline__ RowStat join_row(const SegPart *part, int S, ExpScale c) {
    const int lane = threadIdx.x & 63;
    SegPart x{0., -INFINITY, 0x7FFFFFFF};
    if (lane < S) x = part[lane];
    const float m = wave_max_dpp(x.m);
    double s = 0.;
    if (lane < S) s = x.m == -INFINITY ? x.s : x.s * exp(((double)x.m - (double)m) * c.inv);    // (a segment without any keeps its NaN)
    s = wave_sum_f64(s);
    int id = x.m == m ? x.id : 0x7FFFFFFF;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) id = min(id, __shfl_xor(id, o));
    return RowStat{m, s > 0. && s < INFINITY && m < INFINITY ? 1. / s : 0., id};
}

// The accepted drafts of a request and where its next token comes from: each wave of a
// workgroup takes every fourth draft.
template <typename L> __device__ __forceinline__ Verdict judge(const VerifyParams<L> &p, int r, int n, int first, int &accepted) {
    __shared__ int s_stop;
    __shared__ Verdict s_v;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    if (threadIdx.x == 0) s_stop = n;
    __syncthreads();
    const int targets = p.R * (p.K + 1);
    for (int i = wave; i < n; i += kSegThreads / 64) {
        const RowStat a = join_row(p.part + (int64_t)(r * (p.K + 1) + i) * p.S, p.S, p.c);
        const int y = p.drafts[(int64_t)r * p.K + i];
        bool yes = a.inv > 0. && y < p.V;
        if (p.greedy) {
            yes = yes && y == a.id;
        } else if (yes) {
            const double z = (double)Piece<L>::one(p.z + (first + i) * p.ld + y);
            const double pr = exp((z - (double)a.m) * p.c.inv) * a.inv;
            double q = 1.;
            if (p.d) {
                const RowStat b = join_row(p.part + ((int64_t)targets + r * p.K + i) * p.S, p.S, p.c);
                const double zq = (double)Piece<L>::one(p.d + r * p.ld_request + i * p.ld_draft + y);
                q = exp((zq - (double)b.m) * p.c.inv) * b.inv;
                yes = b.inv > 0.;
            }
            yes = yes && (double)p.u[(int64_t)r * (p.K + 1) + i] * q < pr;
        }
        if (!yes && lane == 0) atomicMin(&s_stop, i);
    }
    __syncthreads();
    const int j = s_stop;
    accepted = j;
    if (wave == 0) {
        const RowStat a = join_row(p.part + (int64_t)(r * (p.K + 1) + j) * p.S, p.S, p.c);
        Verdict v{a.inv, 0., a.m, 0.f, kFromP, first + j};
        if (!(a.inv > 0.)) v.kind = kNone;
        else if (p.greedy) { v.kind = kToken; v.row = a.id; }
        else if (j < n && p.d) {
            const RowStat b = join_row(p.part + ((int64_t)targets + r * p.K + j) * p.S, p.S, p.c);
            v.kind = b.inv > 0. ? kFromRest : kNone;
            v.q_inv = b.inv;
            v.q_m = b.m;
        } else if (j < n) {
            v.kind = kWithout;
        }
        if (lane == 0) s_v = v;
    }
    __syncthreads();
    return s_v;
}
// The mass that id has in what the next token is drawn from.
template <typename L> struct Masses {
    Verdict v; ExpScale c; int without;
    const L *p, *q;
    __device__ __forceinline__ double of(float zp, float zq, int id) const {
        double x = (double)exp_diff(zp, v.p_m, c) * v.p_inv;
        if (v.kind == kFromRest) {
            x -= (double)exp_diff(zq, v.q_m, c) * v.q_inv;
            x = x > 0. ? x : 0.;
        } else if (v.kind == kWithout && id == without) {
            x = 0.;
        }
        return x;
    }
};
template <typename L> __device__ __forceinline__ Masses<L> masses_of(const VerifyParams<L> &p, const Verdict &v, int r, int j) {
    Masses<L> a{v, p.c, -1, p.z + v.row * p.ld, nullptr};
    if (v.kind == kFromRest) a.q = p.d + r * p.ld_request + j * p.ld_draft;
    if (v.kind == kWithout) a.without = p.drafts[(int64_t)r * p.K + j];
    return a;
}
// A thread's masses of its elements of a segment, in turn.
template <typename L, typename F> __device__ __forceinline__ void each_mass(const Masses<L> &a, int lo, int n, F f) {
    float z[kSegEach];
    each_of(a.p, lo, n, [&](float x, int, int k) { z[k] = x; });
    if (a.q) {
        each_of(a.q, lo, n, [&](float x, int id, int k) { f(a.of(z[k], x, id), id, k); });
    } else {
        constexpr int N = Piece<L>::N;
#pragma unroll
        for (int k = 0; k < kSegEach; ++k) {
            const int id = lo + ((int)threadIdx.x + k / N * kSegThreads) * N + k % N;
            f(a.of(z[k], 0.f, id), id, k);
        }
    }
}

template <typename L> __global__ __launch_bounds__(kSegThreads) void k_verify_masses(VerifyParams<L> p) {
    __shared__ double s_s[kSegThreads / 64];
    const int seg = blockIdx.x % p.S, r = blockIdx.x / p.S;
    int first, j;
    const int n = rows_of(p, r, first);
    if (n < 0) {
        if (seg == 0 && threadIdx.x == 0) {
            p.verdict[r] = Verdict{0., 0., 0.f, 0.f, kNone, 0};
            p.accepted[r] = 0;
        }
        return;
    }
    const Verdict v = judge(p, r, n, first, j);
    if (seg == 0 && threadIdx.x == 0) {
        p.verdict[r] = v;
        p.accepted[r] = j;
    }
    if (v.kind == kNone || v.kind == kToken) return;
    const Masses<L> a = masses_of(p, v, r, j);
    const int lo = seg * kSeg;
    double s = 0.;
    each_mass(a, lo, min(kSeg, p.V - lo), [&](double x, int, int) { s += x; });
    s = block_sum<kSegThreads>(s, s_s);
    if (threadIdx.x == 0) p.mass[(int64_t)r * p.S + seg] = s;
}

template <typename L> __global__ __launch_bounds__(kSegThreads) void k_verify_tokens(VerifyParams<L> p) {
    constexpr int W = kSegThreads / 64, N = Piece<L>::N, P = kSegEach / N;
    __shared__ double s_sum[P][W];
    __shared__ int s_id, s_last;
    const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const Verdict was = p.verdict[r];
    const int j = p.accepted[r];
    int token = -1;
    if (was.kind == kToken) token = was.row;
    else if (was.kind != kNone) {
        Verdict v = was;
        double mine = lane < p.S ? p.mass[(int64_t)r * p.S + lane] : 0.;
        if (!(wave_sum_f64(mine) > 0.)) {       // p is nowhere above q
            v.kind = kFromP;
            const SegPart x = p.part[(int64_t)(r * (p.K + 1) + j) * p.S + min(lane, p.S - 1)];
            mine = lane < p.S && x.m != -INFINITY ? x.s * exp(((double)x.m - (double)v.p_m) * p.c.inv) * v.p_inv : 0.;
        }
        // the segment at which the running sum exceeds the number's share
        double run = mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const double b = __shfl_up(run, o);
            if (lane >= o) run += b;
        }
        const double all = readlane_f64(run, 63), t = (double)p.u[(int64_t)r * (p.K + 1) + p.K] * all;
        const uint64_t some = __ballot(mine > 0.), over = __ballot(run > t && mine > 0.);
        const int seg = over ? __builtin_ctzll(over) : 63 - __builtin_clzll(some | 1);
        const double before = __shfl(run, seg) - __shfl(mine, seg);
        // its elements: the sums of each round's waves, then of the lanes before this one
        const Masses<L> a = masses_of(p, v, r, j);
        const int lo = seg * kSeg, len = min(kSeg, p.V - lo);
        double x[kSegEach];
        each_mass(a, lo, len, [&](double e, int, int k) { x[k] = e; });
        double in[P];
#pragma unroll
        for (int i = 0; i < P; ++i) {
            double e = 0.;
#pragma unroll
            for (int k = 0; k < N; ++k) e += x[i * N + k];
            in[i] = e;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const double b = __shfl_up(in[i], o);
                if (lane >= o) in[i] += b;
            }
            if (lane == 63) s_sum[i][wave] = in[i];
            in[i] -= e;
        }
        if (tid == 0) { s_id = p.V; s_last = -1; }
        __syncthreads();
        double base = before;
        int found = p.V, last = -1;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            double at = base;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                if (w < wave) at += s_sum[i][w];
                base += s_sum[i][w];
            }
            at += in[i];
#pragma unroll
            for (int k = 0; k < N; ++k) {
                at += x[i * N + k];
                const int id = lo + (tid + i * kSegThreads) * N + k;
                if (x[i * N + k] > 0.) {
                    last = id;
                    if (at > t && id < found) found = id;
                }
            }
        }
        if (found < p.V) atomicMin(&s_id, found);
        if (last >= 0) atomicMax(&s_last, last);
        __syncthreads();
        token = s_id < p.V ? s_id : s_last;     // (rounding may leave the last one's sum short of its share)
    }
    if (tid <= p.K) {
        const int i = tid;
        p.tokens[(int64_t)r * (p.K + 1) + i] = i < j ? p.drafts[(int64_t)r * p.K + i] : i == j ? token : -1;
    }
}
// Greedy: no masses.
template <typename L> __global__ __launch_bounds__(kSegThreads) void k_verify_greedy(VerifyParams<L> p) {
    const int r = blockIdx.x;
    int first, j = 0, token = -1;
    const int n = rows_of(p, r, first);
    if (n >= 0) {
        const Verdict v = judge(p, r, n, first, j);
        if (v.kind == kToken) token = v.row;
    }
    const int i = threadIdx.x;
    if (i == 0) p.accepted[r] = j;
    if (i <= p.K) p.tokens[(int64_t)r * (p.K + 1) + i] = i < j ? p.drafts[(int64_t)r * p.K + i] : i == j ? token : -1;
}

static int segments(int V) { return (V + kSeg - 1) / kSeg; }
static int64_t verify_bytes(int R, int K, int V) {
    const int64_t S = segments(V);
    return (int64_t)R * (2 * K + 1) * S * (int64_t)sizeof(SegPart) + R * S * 8 + (int64_t)R * sizeof(Verdict);
}
static bool verify_sizes_ok(int R, int K, int V) {
    return R >= 0 && R <= 65535 && K >= 0 && K <= 63 && V >= 1 && V <= kOpdMaxVocab &&
           (int64_t)R * (2 * K + 1) * segments(V) < (int64_t)1 << 31;
}

template <typename L>
static int verify(int32_t R, int32_t K, int32_t V, int32_t rows, const L *z, int64_t ld, const int32_t *starts,
                  const int32_t *drafts, const L *d, int64_t ld_request, int64_t ld_draft, const float *u,
                  double temperature, int32_t *tokens, int32_t *accepted, void *work, int64_t work_bytes, void *stream) {
    if (!verify_sizes_ok(R, K, V) || rows < 0 || !(temperature <= 1e5)) return PIPO_EINVAL;
    if (R == 0) return PIPO_OK;
    const bool greedy = temperature <= 0.;
    if (!opd_rows_ok(rows, V, z, ld, greedy ? 1. : temperature, sizeof(L))) return PIPO_EINVAL;
    if (!starts && rows < (int64_t)R * (K + 1)) return PIPO_EINVAL;
    if ((K > 0 && !kv8_aligned(drafts, 4)) || !kv8_aligned(u, 4) || !kv8_aligned(tokens, 4) || !kv8_aligned(accepted, 4) ||
        ((uintptr_t)starts & 3) || !kv8_aligned(work, 16) || work_bytes < verify_bytes(R, K, V))
        return PIPO_EINVAL;
    if (greedy || K == 0) d = nullptr;
    if (d && (!kv8_aligned(d, sizeof(L)) || ld_request < 0 || ld_draft < 0 || ld_request > (int64_t)1 << 40 ||
              ld_draft > (int64_t)1 << 31 || (K > 1 && ld_draft < V) || (R > 1 && ld_request < V)))
        return PIPO_EINVAL;
    VerifyParams<L> p{z, ld, d, ld_request, ld_draft, starts, drafts, u, R, K, V, rows, segments(V), greedy,
                      exp_scale(greedy ? 1. : temperature), tokens, accepted, (SegPart *)work, nullptr, nullptr};
    p.mass = (double *)(p.part + (int64_t)R * (2 * K + 1) * p.S);
    p.verdict = (Verdict *)(p.mass + (int64_t)R * p.S);
    hipStream_t s = (hipStream_t)stream;
    const int64_t lines = (int64_t)R * (K + 1) + (d ? (int64_t)R * K : 0);
    bool ok = launch(k_verify_rows<L>, (unsigned)(lines * p.S), kSegThreads, 0, s, p);
    if (greedy) ok = ok && launch(k_verify_greedy<L>, (unsigned)R, kSegThreads, 0, s, p);
    else ok = ok && launch(k_verify_masses<L>, (unsigned)(R * p.S), kSegThreads, 0, s, p) &&
              launch(k_verify_tokens<L>, (unsigned)R, kSegThreads, 0, s, p);
    return ok ? PIPO_OK : PIPO_EHIP;
}

}  // namespace pipo

using namespace pipo;

extern "C" int64_t pipo_verify_work_bytes(int32_t R, int32_t K, int32_t V) {
    return verify_sizes_ok(R, K, V) && R > 0 ? verify_bytes(R, K, V) : 0;
}
extern "C" int pipo_verify_drafts(int32_t R, int32_t K, int32_t V, int32_t rows, const float *d_logits, int64_t ld,
                                  const int32_t *d_starts, const int32_t *d_drafts, const float *d_draft_logits,
                                  int64_t ld_request, int64_t ld_draft, const float *d_u, double temperature,
                                  int32_t *d_tokens, int32_t *d_accepted, void *d_work, int64_t work_bytes,
                                  void *stream) {
    return verify<float>(R, K, V, rows, d_logits, ld, d_starts, d_drafts, d_draft_logits, ld_request, ld_draft, d_u,
                         temperature, d_tokens, d_accepted, d_work, work_bytes, stream);
}
extern "C" int pipo_verify_drafts_bf16(int32_t R, int32_t K, int32_t V, int32_t rows, const uint16_t *d_logits,
                                       int64_t ld, const int32_t *d_starts, const int32_t *d_drafts,
                                       const uint16_t *d_draft_logits, int64_t ld_request, int64_t ld_draft,
                                       const float *d_u, double temperature, int32_t *d_tokens, int32_t *d_accepted,
                                       void *d_work, int64_t work_bytes, void *stream) {
    return verify<uint16_t>(R, K, V, rows, d_logits, ld, d_starts, d_drafts, d_draft_logits, ld_request, ld_draft, d_u,
                            temperature, d_tokens, d_accepted, d_work, work_bytes, stream);
}
