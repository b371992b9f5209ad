// Verification of drafted tokens against a target's logits from given random numbers.
//
// Draft i of a request is accepted while u_i q_i < p_i; the token behind the accepted ones
// is drawn from max(p - q, 0), or p, by the inverse of its running sum over the ids.
// Two launches: each segment of each row to its maximum and its sum of exponentials of
// differences to it (every logit read once, from HBM: what bounds it); then for each request
// the accepted drafts from a few numbers a row, the masses of the segments of the one or
// two rows that the next token is drawn from (again from the caches), and by the
// workgroup that finishes last the segment that holds the drawn mass, element by
// element.  Exponentials are fp32 of exact differences, masses fp32 products of them
// (added eight, or in fp32 rows four, at a time); sums are added, in a fixed order, and
// compared in 64 bits.
// 64 requests of four drafts over 151936 bf16 logits: 30 us (5.9 TB/s of row bytes) and 20
// (judging 5, two rows a request from the memory-side cache, the draw 5); one request of
// one draft 4 and 9, latency.  Segments of 16384 in the second launch: 22.
#include "kv8.h"

namespace pipo {

constexpr int kSeg = 8192;          // logits of a segment
constexpr int kLine = 32;
constexpr int kRowThreads = 256, kTokenThreads = 512;   // (with 256 too a request's rows take the second launch's waves two turns: 22 us, 64 x 4)
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
    int32_t *done;                  // [R][kLine]: workgroups that have written their mass, a cache line each
};

// Rows of request r: the first, and how many drafts have one (-1: no rows at all).
template <typename L> __device__ __forceinline__ int rows_of(const VerifyParams<L> &p, int r, int &first) {
    RequestRows rr{r * (p.K + 1), p.K + 1};
    if (p.starts) rr = request_rows(p.starts[r], p.starts[r + 1], p.rows);
    first = rr.first;
    return min(rr.n - 1, p.K);
}
// ... of which so many come before the first negative one (up to 63: a lane each).
template <typename L> __device__ __forceinline__ int drafts_of(const VerifyParams<L> &p, int r, int n) {
    const int lane = threadIdx.x & 63;
    return __builtin_ctzll(__ballot(lane >= n || p.drafts[(int64_t)r * p.K + lane] < 0));
}
// The logits of a segment that one of NT threads has: whole pieces, NT apart, and one element of what is left behind
// the last whole one.  Elements that are not there are -inf.
template <typename L, int NT> struct SegRow {
    static constexpr int N = Piece<L>::N, P = kSeg / NT / N;
    u32x4 w[P];
    float tail;
    __device__ __forceinline__ void load(const L *row, int lo, int len) {
#pragma unroll
        for (int k = 0; k < P; ++k) {
            const int e0 = ((int)threadIdx.x + k * NT) * N;
            w[k] = u32x4{Piece<L>::kNegInf, Piece<L>::kNegInf, Piece<L>::kNegInf, Piece<L>::kNegInf};
            if (e0 + N <= len) w[k] = *(const typename Piece<L>::raw_t *)(row + lo + e0);
        }
        tail = -INFINITY;
        if (tail_at(len) < len) tail = Piece<L>::one(row + lo + tail_at(len));
    }
    static __device__ __forceinline__ int tail_at(int len) { return len / N * N + (int)threadIdx.x; }
    static __device__ __forceinline__ int at(int k, int e) { return ((int)threadIdx.x + k * NT) * N + e; }
    __device__ __forceinline__ float get(int k, int e) const { return Piece<L>::get(w[k], e); }
};

template <typename L> __global__ __launch_bounds__(kRowThreads) void k_verify_rows(VerifyParams<L> p) {
    constexpr int N = Piece<L>::N, P = kSeg / kRowThreads / N;
    const int seg = blockIdx.x % p.S, line = blockIdx.x / p.S, targets = p.R * (p.K + 1);
    const bool target = line < targets;
    const int at = target ? line : line - targets, each = target ? p.K + 1 : p.K, r = at / each, i = at - r * each;
    int first;
    const int n = rows_of(p, r, first);
    if (target && i == 0 && seg == 0 && threadIdx.x == 0) p.done[r * kLine] = 0;
    if (target ? i > n : i >= n) return;
    const L *row = target ? p.z + (first + i) * p.ld : p.d + r * p.ld_request + i * p.ld_draft;
    __shared__ float s_m[kRowThreads / 64];
    __shared__ double s_s[kRowThreads / 64];
    __shared__ int s_id[kRowThreads / 64];
    const int lo = seg * kSeg, len = min(kSeg, p.V - lo);
    SegRow<L, kRowThreads> x;
    x.load(row, lo, len);           // (before the drafts, which may say that nobody needs them)
    if (i > drafts_of(p, r, n) - !target) return;
    float m = x.tail;
#pragma unroll
    for (int k = 0; k < P; ++k)
#pragma unroll
        for (int e = 0; e < N; ++e) m = fmaxf(m, x.get(k, e));
    m = block_max<kRowThreads>(m, s_m);
    // (without any token only a NaN is left to be found)
    auto term = [&](float v) { return m == -INFINITY ? v != v ? v : 0.f : exp_diff(v, m, p.c); };
    float sum = term(x.tail);
#pragma unroll
    for (int k = 0; k < P; ++k)
#pragma unroll
        for (int e = 0; e < N; ++e) sum += term(x.get(k, e));
    const double s = block_sum<kRowThreads>((double)sum, s_s);
    int id = p.V;
    if (p.greedy) {
        if (x.tail == m) id = lo + x.tail_at(len);
#pragma unroll
        for (int k = P - 1; k >= 0; --k)
#pragma unroll
            for (int e = N - 1; e >= 0; --e)
                if (x.get(k, e) == m) id = lo + x.at(k, e);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) id = min(id, __shfl_xor(id, o));
        if ((threadIdx.x & 63) == 0) s_id[threadIdx.x >> 6] = id;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kRowThreads / 64; ++k) id = min(id, s_id[k]);
    }
    if (threadIdx.x == 0) p.part[(int64_t)line * p.S + seg] = SegPart{s, m, id};
}

// A row from its segments, in every lane of a wave: maximum, 1 / sum (0: the row is bad), its largest logit's id.
struct RowStat { float m; int id; double inv; };
__device__ __forceinline__ RowStat join_row(const SegPart *part, int S, ExpScale c, bool greedy) {
    const int lane = threadIdx.x & 63;
    SegPart x{0., -INFINITY, 0x7FFFFFFF};
    if (lane < S) x = part[lane];
    const float m = wave_max_dpp(x.m);
    // (a segment without any keeps its NaN)
    const double s = wave_sum_f64(x.m == -INFINITY ? x.s : x.s * (double)exp_diff(x.m, m, c));
    int id = x.m == m ? x.id : 0x7FFFFFFF;
    if (greedy) {
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) id = min(id, __shfl_xor(id, o));
    }
    return RowStat{m, id, s > 0. && s < INFINITY && m < INFINITY ? 1. / s : 0.};
}

// The accepted drafts of a request and where its next token comes from: each wave of a
// workgroup takes every eighth draft, and the row behind them.
template <typename L> __device__ __forceinline__ Verdict judge(const VerifyParams<L> &p, int r, int n, int first, int &accepted) {
    __shared__ int s_stop;
    __shared__ RowStat s_p[64], s_q[64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    if (threadIdx.x == 0) s_stop = n;
    __syncthreads();
    const SegPart *targets = p.part + (int64_t)r * (p.K + 1) * p.S, *drawn = p.part + ((int64_t)p.R * (p.K + 1) + r * p.K) * p.S;
    for (int i = wave; i <= n; i += kTokenThreads / 64) {
        const int y = i < n ? p.drafts[(int64_t)r * p.K + i] : 0;
        const bool in = i < n && y < p.V;
        const float u = p.u[(int64_t)r * (p.K + 1) + i];
        const float z = in && !p.greedy ? Piece<L>::one(p.z + (first + i) * p.ld + y) : 0.f;
        const float zq = in && p.d ? Piece<L>::one(p.d + r * p.ld_request + i * p.ld_draft + y) : 0.f;
        const RowStat a = join_row(targets + i * p.S, p.S, p.c, p.greedy);
        RowStat b{0.f, 0, 0.};
        if (p.d && i < n) b = join_row(drawn + i * p.S, p.S, p.c, false);
        bool yes = in && a.inv > 0.;
        if (p.greedy) {
            yes = yes && y == a.id;
        } else if (yes) {
            const double q = p.d ? (double)exp_diff(zq, b.m, p.c) * b.inv : 1.;
            yes = (!p.d || b.inv > 0.) && (double)u * q < (double)exp_diff(z, a.m, p.c) * a.inv;
        }
        if (lane == 0) {
            s_p[i] = a;
            s_q[i] = b;
            if (i < n && !yes) atomicMin(&s_stop, i);
        }
    }
    __syncthreads();
    const int j = s_stop;
    accepted = j;
    const RowStat a = s_p[j], b = s_q[j];
    Verdict v{a.inv, b.inv, a.m, b.m, kFromP, first + j};
    if (!(a.inv > 0.)) v.kind = kNone;
    else if (p.greedy) { v.kind = kToken; v.row = a.id; }
    else if (j < n && p.d) v.kind = b.inv > 0. ? kFromRest : kNone;
    else if (j < n) v.kind = kWithout;
    return v;
}
template <typename L> __device__ __forceinline__ void put_tokens(const VerifyParams<L> &p, int r, int j, int token) {
    const int i = threadIdx.x;
    if (i == 0) p.accepted[r] = j;
    if (i <= p.K) p.tokens[(int64_t)r * (p.K + 1) + i] = i < j ? p.drafts[(int64_t)r * p.K + i] : i == j ? token : -1;
}
// What the next token is drawn from: the masses of a thread's logits of a segment.
template <typename L> struct Masses {
    Verdict v; ExpScale c; int without, lo, len;
    typedef SegRow<L, kTokenThreads> Row;
    Row p, q;
    __device__ __forceinline__ Masses(const VerifyParams<L> &a, const Verdict &v_, int r, int j, int seg)
        : v(v_), c(a.c), without(-1), lo(seg * kSeg), len(min(kSeg, a.V - seg * kSeg)) {
        p.load(a.z + v.row * a.ld, lo, len);
        if (v.kind == kFromRest) q.load(a.d + r * a.ld_request + j * a.ld_draft, lo, len);
        if (v.kind == kWithout) without = a.drafts[(int64_t)r * a.K + j] - lo;
    }
    __device__ __forceinline__ float of(float zp, float zq, int at) const {
        const float x = exp_diff(zp, v.p_m, c) * (float)v.p_inv;
        if (v.kind == kFromRest) return fmaxf(fmaf(exp_diff(zq, v.q_m, c), -(float)v.q_inv, x), 0.f);
        return at == without ? 0.f : x;
    }
    __device__ __forceinline__ float get(int k, int e) const { return of(p.get(k, e), q.get(k, e), p.at(k, e)); }
    __device__ __forceinline__ float piece(int k) const {
        float s = get(k, 0);
#pragma unroll
        for (int e = 1; e < Row::N; ++e) s += get(k, e);
        return s;
    }
    __device__ __forceinline__ float tail() const { return of(p.tail, q.tail, p.tail_at(len)); }
};

// Running sums over the lanes by DPP: within each row of 16, then the rows before.
template <int CTRL, int ROWS> __device__ __forceinline__ double shifted_f64(double v) {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);     // (0 where there is no lane to take from)
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, ROWS, 0xF, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, ROWS, 0xF, false);
    return __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}
__device__ __forceinline__ double wave_scan_f64(double v) {
    v += shifted_f64<0x111, 0xF>(v);    // row_shr 1, 2, 4, 8
    v += shifted_f64<0x112, 0xF>(v);
    v += shifted_f64<0x114, 0xF>(v);
    v += shifted_f64<0x118, 0xF>(v);
    v += shifted_f64<0x142, 0xA>(v);    // lane 15 of the first and third row to the next
    v += shifted_f64<0x143, 0xC>(v);    // lane 31 to the last two rows
    return v;
}
// Of 64 masses in order, a lane each: the first at which the running sum from `from` on
// exceeds t, or (rounding, or a number that is none) the last that is positive; `from`
// becomes the sum before it.
__device__ __forceinline__ int crossing(double mine, double t, double &from) {
    const double run = wave_scan_f64(mine);
    const uint64_t some = __ballot(mine > 0.), over = __ballot(from + run > t && mine > 0.);
    const int at = over ? __builtin_ctzll(over) : 63 - __builtin_clzll(some | 1);
    from += readlane_f64(run, at) - readlane_f64(mine, at);
    return at;
}
// The token at which the running sum of a request's masses exceeds its number's share.
template <typename L> __device__ __forceinline__ int draw_token(const VerifyParams<L> &p, Verdict v, int r, int j) {
    constexpr int W = kTokenThreads / 64, N = Piece<L>::N, P = kSeg / kTokenThreads / N;
    static_assert((P + 1) * W <= 64, "a lane for each wave and round");
    __shared__ double s_sum[(P + 1) * W];
    __shared__ int s_token;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    double mine = 0.;
    if (lane < p.S) mine = __hip_atomic_load(p.mass + (int64_t)r * p.S + lane, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const double u = (double)p.u[(int64_t)r * (p.K + 1) + p.K];
    double all = wave_sum_f64(mine);
    if (!(all > 0.)) {              // p is nowhere above q
        v.kind = kFromP;
        const SegPart x = p.part[(int64_t)(r * (p.K + 1) + j) * p.S + min(lane, p.S - 1)];
        mine = lane < p.S && x.m != -INFINITY ? x.s * (double)exp_diff(x.m, v.p_m, p.c) * v.p_inv : 0.;
        all = wave_sum_f64(mine);
    }
    const double t = u * all;
    double from = 0.;
    const int seg = crossing(mine, t, from);
    // its elements by rounds of the workgroup's threads (the last: what is left behind the whole pieces) and waves
    const Masses<L> x(p, v, r, j, seg);
    double in[P + 1];
#pragma unroll
    for (int i = 0; i <= P; ++i) {
        in[i] = i == P ? x.tail() : x.piece(i);
        const double sum = wave_sum_f64(in[i]);
        if (lane == 0) s_sum[i * W + wave] = sum;
    }
    __syncthreads();
    const int part = crossing(lane < (P + 1) * W ? s_sum[lane] : 0., t, from);
    if (part % W == wave) {         // this wave has it: its lanes, then the lane's elements
        double e = 0.;
#pragma unroll
        for (int i = 0; i <= P; ++i) e = part / W == i ? in[i] : e;
        const int l = crossing(e, t, from);
        int id = p.V - 1;
        if (lane == l) {
            bool found = false;
#pragma unroll
            for (int i = 0; i <= P; ++i) {
                if (part / W != i) continue;
                auto next = [&](float m, int at) {
                    from += (double)m;
                    if (m > 0.f && !found) {
                        id = x.lo + at;
                        found = from > t;
                    }
                };
                if (i == P) next(x.tail(), x.p.tail_at(x.len));
                else {
#pragma unroll
                    for (int k = 0; k < N; ++k) next(x.get(i, k), x.p.at(i, k));
                }
            }
            s_token = id;
        }
    }
    __syncthreads();
    return s_token;
}

template <typename L> __global__ __launch_bounds__(kTokenThreads) void k_verify_tokens(VerifyParams<L> p) {
    __shared__ double s_s[kTokenThreads / 64];
    __shared__ int s_done;
    const int seg = p.greedy ? 0 : blockIdx.x % p.S, r = p.greedy ? blockIdx.x : blockIdx.x / p.S;
    int first, j = 0;
    const int n = rows_of(p, r, first);
    Verdict v{0., 0., 0.f, 0.f, kNone, 0};
    if (n >= 0) v = judge(p, r, drafts_of(p, r, n), first, j);
    if (v.kind == kNone || v.kind == kToken) {
        if (seg == 0) put_tokens(p, r, j, v.kind == kToken ? v.row : -1);
        return;
    }
    const Masses<L> x(p, v, r, j, seg);
    double s = x.tail();
#pragma unroll
    for (int k = 0; k < Masses<L>::Row::P; ++k) s += (double)x.piece(k);
    s = block_sum<kTokenThreads>(s, s_s);
    // the last to have written its mass goes on (the first launch has cleared the count)
    if (threadIdx.x == 0) {
        __hip_atomic_store(p.mass + (int64_t)r * p.S + seg, s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        // (both are agent-wide by themselves and the one is there before the other: no cache has to be written back)
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        s_done = __hip_atomic_fetch_add(p.done + r * kLine, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (s_done != p.S - 1) return;
    put_tokens(p, r, j, draw_token(p, v, r, j));
}

static int segments(int V) { return (V + kSeg - 1) / kSeg; }
static int64_t verify_bytes(int R, int K, int V) {
    const int64_t S = segments(V);
    return (int64_t)R * (2 * K + 1) * S * (int64_t)sizeof(SegPart) + R * S * 8 + (int64_t)R * kLine * 4;
}
static bool verify_sizes_ok(int R, int K, int V) {
    return R >= 0 && R <= 65535 && K >= 0 && K <= 63 && V >= 1 && V <= kOpdMaxVocab &&
           (int64_t)R * (2 * K + 1) * segments(V) < (int64_t)1 << 24;      // (a launch's threads are counted in 32 bits)
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
    p.done = (int32_t *)(p.mass + (int64_t)R * p.S);
    hipStream_t s = (hipStream_t)stream;
    const int64_t lines = (int64_t)R * (K + 1) + (d ? (int64_t)R * K : 0);
    const bool ok = launch(k_verify_rows<L>, (unsigned)(lines * p.S), kRowThreads, 0, s, p) &&
                    launch(k_verify_tokens<L>, (unsigned)(greedy ? R : R * p.S), kTokenThreads, 0, s, p);
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
