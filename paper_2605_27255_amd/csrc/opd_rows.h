// Logit rows of the OPD operators: 16-byte pieces at any element alignment,
// exponentials of differences at a temperature, and sums of them that carry
// their own maximum.
#pragma once
#include "device_common.h"
#include <math.h>

namespace pipo {

constexpr double kLn2 = 0.69314718055994530942;
constexpr int kOpdMaxVocab = 1 << 19;
constexpr int kMaxParts = 64;       // workgroups of a split row: a lane of a wave joins each
struct Part { float m, B; double s; int bad, pad; };     // what a segment of a row leaves for the others (a RowSum)

// ---- launches and checks on the host, shared by the entry points ---------------------
// (the launch's own status: asking for the last error takes another microsecond)
template <typename... A, typename... B>
inline bool launch(void (*kernel)(A...), unsigned grid, unsigned block, size_t lds, hipStream_t s, B... args) {
    void *ptrs[] = {(void *)&args...};
    return hipLaunchKernel((const void *)kernel, dim3(grid), dim3(block), ptrs, lds, s) == hipSuccess;
}
bool opd_rows_ok(int32_t T, int32_t V, const void *z, int64_t ld, double temperature, size_t es);
bool opd_work_ok(const void *work, int64_t work_bytes, int64_t need);
int64_t opd_loss_work_bytes(int T, int V, int k, int es, bool grad);

// ---- pieces of 16 bytes of a row ------------------------------------------------
// A row may start at any multiple of its element (odd vocabularies, padded or
// sliced rows); 16-byte accesses across the grid of 16 are slow (512 x 50021 bf16
// rows with their gradient: 35 us, from aligned pieces 24).  So its pieces lie on
// the grid: piece 0 starts `head` elements into the row, and what is before it
// (piece -1) and behind the last whole one are partial pieces, taken element by
// element.
template <typename L> struct Piece;
template <> struct Piece<float> {
    static constexpr int N = 4;
    typedef u32x4 __attribute__((aligned(4))) raw_t;     // (a gradient's rows need not lie like the logits')
    static __device__ __forceinline__ float get(u32x4 w, int e) { return __uint_as_float(w[e]); }
    static __device__ __forceinline__ u32x4 pack(const float *v) {
        return u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    }
    static __device__ __forceinline__ float one(const float *p) { return *p; }
    static __device__ __forceinline__ void put(float *p, float v) { *p = v; }
    static constexpr uint32_t kNegInf = 0xFF800000u;
};
template <> struct Piece<uint16_t> {
    static constexpr int N = 8;
    typedef u32x4 __attribute__((aligned(2))) raw_t;
    static __device__ __forceinline__ float get(u32x4 w, int e) { return (e & 1) ? bf_hi(w[e >> 1]) : bf_lo(w[e >> 1]); }
    static __device__ __forceinline__ u32x4 pack(const float *v) {
        return u32x4{pack_bf2_hw(v[0], v[1]), pack_bf2_hw(v[2], v[3]), pack_bf2_hw(v[4], v[5]), pack_bf2_hw(v[6], v[7])};
    }
    static __device__ __forceinline__ float one(const uint16_t *p) { return bf2f(*p); }
    static __device__ __forceinline__ void put(uint16_t *p, float v) { *p = (uint16_t)pack_bf2_hw(v, 0.f); }
    static constexpr uint32_t kNegInf = 0xFF80FF80u;
};

template <typename L> struct Span {
    L *body;                        // piece 0
    int head, n, whole;             // elements before piece 0, elements in all, whole pieces
    __device__ __forceinline__ Span(L *row, int n_) : n(n_) {
        constexpr int es = sizeof(L);
        head = min((int)((16 - ((uintptr_t)row & 15)) & 15) / es, n);
        body = row + head;
        whole = (n - head) / (16 / es);
    }
    // no partial pieces (the same for the whole workgroup)
    __device__ __forceinline__ bool exact() const { return head == 0 && whole * (int)(16 / sizeof(L)) == n; }
    __device__ __forceinline__ bool has(int i, int e) const {   // element e of piece i
        const int at = i * (int)(16 / sizeof(L)) + e;
        return at >= -head && at < n - head;
    }
};
// The fewest whole pieces that one of the rows has.
template <typename L> inline int least_whole(const L *z, int64_t ld, int T, int n) {
    constexpr int N = 16 / sizeof(L);
    if (((uintptr_t)z & 15) == 0 && (T == 1 || ld % N == 0)) return n / N;
    return n < N ? 0 : (n - N + 1) / N;
}

// Piece i, whole.  AGAIN: it is read twice, and may stay in the caches.
template <typename L, bool AGAIN = false> __device__ __forceinline__ u32x4 load_piece(const L *body, int i) {
    const typename Piece<L>::raw_t *at = (const typename Piece<L>::raw_t *)(body + (int64_t)i * Piece<L>::N);
    if (AGAIN) return *at;
    return __builtin_nontemporal_load(at);
}
template <typename L> __device__ __forceinline__ void store_piece(L *body, int i, const float *v) {
    __builtin_nontemporal_store(Piece<L>::pack(v), (typename Piece<L>::raw_t *)(body + (int64_t)i * Piece<L>::N));
}
// The same by byte offset from the row's start, for unrolled walks: with the
// offset in a register that the compiler cannot see through (next_slab), it does
// not keep an address for every step.
template <typename L> __device__ __forceinline__ u32x4 load_at(const L *row, uint32_t off) {
    return __builtin_nontemporal_load((const typename Piece<L>::raw_t *)((const char *)row + off));
}
template <typename L> __device__ __forceinline__ void store_at(L *row, uint32_t off, const float *v) {
    __builtin_nontemporal_store(Piece<L>::pack(v), (typename Piece<L>::raw_t *)((char *)row + off));
}
template <int NT> __device__ __forceinline__ void next_slab(uint32_t &off) {
    off += NT * 16;
    asm volatile("" : "+v"(off));
    __builtin_amdgcn_sched_barrier(0);  // nor mixes the steps, whose temporaries would not fit beside the row
}
// A partial piece: elements outside the row read as -inf and are not written.
// (out: where a gradient's piece 0 lies.)
template <typename L> __device__ __forceinline__ u32x4 load_edge(const Span<const L> &row, int i) {
    typedef Piece<L> P;
    u32x4 w{P::kNegInf, P::kNegInf, P::kNegInf, P::kNegInf};
#pragma unroll
    for (int e = 0; e < P::N; ++e) {
        if (!row.has(i, e)) continue;
        const int at = i * P::N + e;
        if (sizeof(L) == 4) w[e] = ((const uint32_t *)row.body)[at];
        else if (e & 1) w[e >> 1] = (w[e >> 1] & 0xFFFFu) | ((uint32_t)((const uint16_t *)row.body)[at] << 16);
        else w[e >> 1] = (w[e >> 1] & 0xFFFF0000u) | ((const uint16_t *)row.body)[at];
    }
    return w;
}
template <typename L, typename S> __device__ __forceinline__ void store_edge(L *out, const Span<S> &row, int i, const float *v) {
#pragma unroll
    for (int e = 0; e < Piece<L>::N; ++e)
        if (row.has(i, e)) Piece<L>::put(out + i * Piece<L>::N + e, v[e]);
}
// Calls f(piece, its index) for this thread's whole pieces from index first up to
// end, NT apart and U of them in flight.
template <int NT, int U, bool AGAIN = false, typename L, typename F>
__device__ __forceinline__ void whole_pieces(const L *body, int first, int end, F f) {
    int i = first;
    for (; i + (U - 1) * NT < end; i += U * NT) {
        u32x4 w[U];
#pragma unroll
        for (int u = 0; u < U; ++u) w[u] = load_piece<L, AGAIN>(body, i + u * NT);
#pragma unroll
        for (int u = 0; u < U; ++u) f(w[u], i + u * NT);
    }
    for (; i < end; i += NT) f(load_piece<L, AGAIN>(body, i), i);
}
// ... and calls edge(piece, its index) for the partial ones, which belong to the last two threads.
template <int NT, typename L, typename F> __device__ __forceinline__ void edges(const Span<const L> &row, F edge) {
    if (row.exact() || (int)threadIdx.x < NT - 2) return;
    const int i = (int)threadIdx.x == NT - 1 ? -1 : row.whole;
    edge(load_edge(row, i), i);     // (empty where only the other one is there)
}
template <int NT, int U, bool AGAIN = false, typename L, typename F>
__device__ __forceinline__ void each_piece(const Span<const L> &row, int first, F f) {
    whole_pieces<NT, U, AGAIN>(row.body, first, row.whole, f);
    edges<NT>(row, f);
}

// ---- exp(z / temperature) over a reference -------------------------------------------
// 2^(z c - B) with c = log2(e) / temperature in two floats, c rounded down and
// the (positive) rest: one float of c would tilt every term of a sum the same way
// by up to 2^-24 of its exponent, which does not average out.  B is a float known
// exactly, so its own rounding costs nothing.  z = -inf gives 0, a NaN stays one.
struct ExpScale { float hi, lo; double inv; };
inline ExpScale exp_scale(double temperature) {
    const double c = 1.4426950408889634074 / temperature;
    float hi = (float)c;
    if ((double)hi > c) hi = nextafterf(hi, 0.f);
    const float lo = (float)(c - (double)hi);
    return ExpScale{hi, lo > 1e-30f ? lo : 1e-30f, 1.0 / temperature};
}
__device__ __forceinline__ float exp_at(float z, float B, ExpScale c) {
    return __builtin_amdgcn_exp2f(fmaf(z, c.lo, fmaf(z, c.hi, -B)));
}
// Exponents z c beyond this in magnitude are far: there the reference m c.hi is
// rounded by up to a quarter, and further out by as many binades as a sum of floats
// cannot hold.  Far values below near ones (masks, as a rule) weigh nothing; a row of
// nothing nearer, or of far large ones, is summed by differences of its logits
// (exp_diff), which are exact wherever its zero is.
constexpr float kFar = 4194304.f;
__device__ __forceinline__ float ref_of(float m, ExpScale c) {
#pragma clang fp contract(off)      // the product as the one float that every use of it takes
    return fmaxf(m * c.hi, -kFar);
}
__device__ __forceinline__ bool is_far(float m, ExpScale c) { return m != -INFINITY && !(fabsf(m * c.hi) <= kFar); }
__device__ __forceinline__ float exp_diff(float a, float b, ExpScale c) {
    const float d = a - b;
    return __builtin_amdgcn_exp2f(fmaf(d, c.hi, d * c.lo));
}

// ---- (max, sum of 2^(z c - ref_of(max))) ----------------------------------------------
// (S: float, or double where the registers allow it)
template <typename S> struct MaxSum { float m; S s; };
template <int N, typename S> __device__ __forceinline__ void add_values(MaxSum<S> &a, const float *v, ExpScale c) {
    float m = v[0];
#pragma unroll
    for (int e = 1; e < N; ++e) m = fmaxf(m, v[e]);
    if (m > a.m) {
        a.s *= __builtin_amdgcn_exp2f(ref_of(a.m, c) - ref_of(m, c));
        a.m = m;
    }
    const float B = ref_of(a.m, c);
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < N; ++e) s += exp_at(v[e], B, c);
    a.s += s;
}
// ---- reductions without LDS traffic inside a wave ------------------------------------------
// DPP within each row of 16 lanes (pairs, quads, half rows, rows), then the four
// rows' values through scalar registers; every lane gets the result, added in
// the same order in every lane.
__device__ __forceinline__ float wave_max_dpp(float v) {
    v = fmaxf(v, PIPO_DPP(v, 0xB1));
    v = fmaxf(v, PIPO_DPP(v, 0x4E));
    v = fmaxf(v, PIPO_DPP(v, 0x141));
    v = fmaxf(v, PIPO_DPP(v, 0x140));
    const int u = __float_as_int(v);
    return fmaxf(fmaxf(__int_as_float(__builtin_amdgcn_readlane(u, 0)), __int_as_float(__builtin_amdgcn_readlane(u, 16))),
                 fmaxf(__int_as_float(__builtin_amdgcn_readlane(u, 32)), __int_as_float(__builtin_amdgcn_readlane(u, 48))));
}
template <int CTRL> __device__ __forceinline__ double dpp_f64(double v) {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_mov_dpp((int)(uint32_t)u, CTRL, 0xF, 0xF, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_mov_dpp((int)(uint32_t)(u >> 32), CTRL, 0xF, 0xF, false);
    return __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}
__device__ __forceinline__ double readlane_f64(double v, int lane) {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, lane);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), lane);
    return __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}
__device__ __forceinline__ double wave_sum_f64(double v) {
    v += dpp_f64<0xB1>(v);
    v += dpp_f64<0x4E>(v);
    v += dpp_f64<0x141>(v);
    v += dpp_f64<0x140>(v);
    return (readlane_f64(v, 0) + readlane_f64(v, 16)) + (readlane_f64(v, 32) + readlane_f64(v, 48));
}

// ---- over a workgroup of NT threads, in a fixed order; every thread gets the result ----------
// (a value per wave in s_w[NT / 64]; ends with every wave past its reads of what it wrote before)
template <int NT> __device__ __forceinline__ float block_max(float v, float *s_w) {
    v = wave_max_dpp(v);
    if ((threadIdx.x & 63) == 0) s_w[threadIdx.x >> 6] = v;
    __syncthreads();
    v = s_w[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) v = fmaxf(v, s_w[w]);
    return v;
}
template <int NT> __device__ __forceinline__ double block_sum(double v, double *s_w) {
    v = wave_sum_f64(v);
    if ((threadIdx.x & 63) == 0) s_w[threadIdx.x >> 6] = v;
    __syncthreads();
    double r = 0.;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) r += s_w[w];
    return r;
}
// A row's unlisted values: their sum in multiples of 2^B (where m is far, of
// exp(m / temperature)); m is their maximum, or near it (-inf: there are none).
struct RowSum { float m, B; double s; };
// The log of what such a sum counts in over exp(at / temperature).
__device__ __forceinline__ double log_unit(float m, float B, double at, ExpScale c) {
    return is_far(m, c) ? ((double)m - at) * c.inv : (double)B * kLn2 - at * c.inv;
}

// What a workgroup's maxima and sums of a value per wave pass through.
template <int NT> struct Reduce { float max[2][NT / 64]; double sum[2][NT / 64]; };
// The threads' (max, sum) as one.
template <int NT> __device__ __forceinline__ RowSum block_merge(MaxSum<double> a, ExpScale c, Reduce<NT> &red) {
    const float m = block_max<NT>(a.m, red.max[0]);
    const float B = ref_of(m, c);
    return RowSum{m, B, block_sum<NT>(a.s * __builtin_amdgcn_exp2f(ref_of(a.m, c) - B), red.sum[0])};
}

// A row's segments as one (max, sum), in every lane.
__device__ __forceinline__ RowSum join_parts(const Part *part, int S, ExpScale c, bool &bad) {
    const int lane = threadIdx.x & 63;
    Part x{-INFINITY, -kFar, 0., 0, 0};
    if (lane < S) x = part[lane];
    bad = __ballot(x.bad != 0) != 0;
    const float m = wave_max_dpp(x.m);
    const float B = ref_of(m, c);
    // a segment's unit over the row's
    double f = exp(log_unit(x.m, x.B, m, c) - (is_far(m, c) ? 0. : log_unit(m, B, m, c)));
    // nothing there (s is 0, or a NaN that stays): its reference may be far below the others', or above them where all are empty
    if (x.m == -INFINITY || x.m == m) f = 1.;
    return RowSum{m, B, wave_sum_f64(x.s * f)};
}

}  // namespace pipo
