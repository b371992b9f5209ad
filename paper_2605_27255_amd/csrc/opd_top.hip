// The k largest logits of each row, in the order of (value descending, id
// ascending), with their log-probabilities and the log of the mass outside.
//
// One pass over the row: every thread keeps the maximum and the sum of
// exponentials of its own pieces.  A value that at least k threads' maxima
// reach is a lower bound of the k-th largest logit, so only those threads'
// pieces can hold the k largest: they are read again (about k of 1024 threads,
// from the caches), and what reaches the bound, usually little more than k
// values, is ranked by counting.  Threads that hold none of the k keep their
// sums; the others' are added up again without them, so that the mass outside
// the list is a sum of what is outside, not a difference.
// Rows whose values crowd at the bound (constant rows, long ties) overflow the
// candidate array; a radix select over (value, id) keys, which are all
// different, then narrows the row to what fits.
// HBM-bound: V logits read per row.
#include "opd_rows.h"
#include "pipo.h"

namespace pipo {

constexpr int kTopMax = 256;        // k
constexpr int kTopCand = 2048;      // candidates ranked

constexpr double kLn2 = 0.69314718055994530942;

bool opd_rows_ok(int32_t T, int32_t V, const void *z, int64_t ld, double temperature, size_t es);

template <typename L> struct TopParams {
    const L *z; int64_t ld;
    int T, V, k;
    ExpScale c;
    int32_t *ids; float *logp, *tail;
};

// Unsigned integers in the order of the values; -0 counts as 0.
__device__ __forceinline__ uint32_t value_key(float v) {
    const uint32_t u = __float_as_uint(v + 0.f);
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) {
    return __uint_as_float((k & 0x80000000u) ? k & 0x7FFFFFFFu : ~k);
}
// (value, id) keys: all different, larger for larger values and then for lower ids.
__device__ __forceinline__ uint64_t pair_key(uint32_t vkey, int id) {
    return ((uint64_t)vkey << 32) | (uint32_t)~(uint32_t)id;
}
__device__ __forceinline__ int key_id(uint64_t k) { return (int)~(uint32_t)k; }

template <int NT> struct TopShared {
    uint32_t tmax[NT];              // each thread's largest value key, 0: no pieces
    uint64_t cand[kTopCand];
    uint64_t sorted[kTopCand];
    float red[3][NT / 64];
    uint32_t wmin[NT / 64];
    int count[2][NT / 64], wcount[NT / 64];
    int hist[256];
    int n, bin, above;
};

// A bound that at least k of the NT keys reach, and few more: each round every
// wave counts the keys at or above a pivot of its own, so a round cuts the range
// by the number of waves plus one.  lo is reached by at least k, none is above hi.
template <int NT>
__device__ __forceinline__ uint32_t bound_of_kth(TopShared<NT> &sh, uint32_t lo, uint32_t hi, int k) {
    constexpr int W = NT / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t key[W];
#pragma unroll
    for (int i = 0; i < W; ++i) key[i] = sh.tmax[i * 64 + lane];
    for (int round = 0; lo < hi; ++round) {
        const uint64_t span = (uint64_t)(hi - lo) + 1;
        const uint32_t pivot = lo + (uint32_t)(span * (wave + 1) / (W + 1));
        int n = 0;
#pragma unroll
        for (int i = 0; i < W; ++i) n += __popcll(__ballot(key[i] >= pivot));
        int *count = sh.count[round & 1];   // the other half is still read
        if (lane == 0) count[wave] = n;
        __syncthreads();
        // counts fall with the pivot: the last wave whose pivot k keys reach, and the one after it
        const int c = count[lane & (W - 1)];
        const int reach = __popcll(__ballot(lane < W && c >= k));
        const uint32_t base = lo;
        if (reach < W) hi = base + (uint32_t)(span * (reach + 1) / (W + 1)) - 1;
        if (reach > 0) {
            lo = base + (uint32_t)(span * reach / (W + 1));
            if (__builtin_amdgcn_readlane(c, reach - 1) <= k + (k >> 2) + 8) break;
        }
    }
    return lo;
}

template <typename L, int NT>
__global__ __launch_bounds__(NT, 8) void k_opd_top(TopParams<L> p) {
    constexpr int N = Piece<L>::N, W = NT / 64;
    __shared__ TopShared<NT> sh;
    const int t = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int V = p.V, k = p.k, n = (V + N - 1) / N;
    const L *row = p.z + (int64_t)t * p.ld;

    MaxSum own{-INFINITY, 0.f};
    each_piece<NT, 4>(row, tid, V, [&](u32x4 w, int) {
        float v[N];
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = Piece<L>::get(w, e);
        add_values<N>(own, v, p.c);
    });
    const uint32_t mine = tid < n ? value_key(own.m) : 0u;
    sh.tmax[tid] = mine;
    // the least of them, as the largest of the negated maxima (-0 and 0 have one key)
    const float least_w = -wave_max_dpp(tid < n ? -own.m : -INFINITY);
    if (lane == 0) sh.wmin[wave] = value_key(least_w);
    if (tid == 0) sh.n = 0;
    const MaxSum all = block_merge<NT>(own, p.c, sh.red);   // its barrier: tmax, wmin and n are set
    const bool far = is_far(all.m);
    const float B = ref_of(all.m, p.c);
    auto term = [&](float v) { return far ? exp_diff(v, all.m, p.c) : exp_at(v, B, p.c); };
    uint32_t least = sh.wmin[0];
#pragma unroll
    for (int w = 1; w < W; ++w) least = min(least, sh.wmin[w]);
    // fewer pieces than k: everything is a candidate
    const uint32_t bound = n < k ? 0u : bound_of_kth<NT>(sh, least, value_key(all.m), k);

    // the pieces of the threads that reach the bound, again
    const bool picked = mine >= bound && tid < n;
    const uint64_t ball = __ballot(picked);
    if (lane == 0) sh.wcount[wave] = __popcll(ball);
    __syncthreads();                // every wave is past the search: its keys become the picked threads
    int at = 0, total = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        const int c = sh.wcount[w];
        if (w < wave) at += c;
        total += c;
    }
    uint32_t *list = sh.tmax;
    if (picked) list[at + __popcll(ball & ((1ull << lane) - 1))] = tid;
    __syncthreads();
    float rest = picked ? 0.f : own.s * __builtin_amdgcn_exp2f(ref_of(own.m, p.c) - B);
    const int per = (n + NT - 1) / NT;
    for (int x = tid; x < total * per; x += NT) {
        const int i = (int)list[x / per] + NT * (x % per);
        if (i >= n) continue;
        const u32x4 w = i < V / N ? load_piece(row, i) : load_last(row, i, V);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float v = Piece<L>::get(w, e);
            const uint32_t key = value_key(v);
            if (key >= bound && i * N + e < V) {
                const int c = atomicAdd(&sh.n, 1);
                if (c < kTopCand) sh.cand[c] = pair_key(key, i * N + e);
            } else {
                rest += term(v);
            }
        }
    }
    __syncthreads();
    int nc = sh.n;
    if (nc > kTopCand || nc < k || far) {   // too many (ties), or NaNs, which no maximum sees, or sums that do not fit:
                                            // select among all keys
        uint64_t thr = 0;           // keys at or above thr, of which the first `bits` bits are settled
        int need = k;
        for (int bits = 8; bits <= 64; bits += 8) {
            const int sh_bits = 64 - bits;
            __syncthreads();
            for (int i = tid; i < 256; i += NT) sh.hist[i] = 0;
            __syncthreads();
            each_piece<NT, 4>(row, tid, V, [&](u32x4 w, int i) {
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    if (i * N + e >= V) continue;
                    const uint64_t key = pair_key(value_key(Piece<L>::get(w, e)), i * N + e);
                    if (bits > 8 && (key >> (sh_bits + 8)) != (thr >> (sh_bits + 8))) continue;
                    const int bin = (int)(key >> sh_bits) & 255;
                    // values of a crowded row share their bins: one addition for a wave of equal ones
                    const uint64_t same = __ballot(bin == __builtin_amdgcn_readfirstlane(bin));
                    if (same == __ballot(1)) {
                        if (lane == (int)__builtin_ctzll(same)) atomicAdd(&sh.hist[bin], __popcll(same));
                    } else {
                        atomicAdd(&sh.hist[bin], 1);
                    }
                }
            });
            __syncthreads();
            if (tid == 0) {
                int b = 255, above = 0;
                while (b > 0 && above + sh.hist[b] < need) above += sh.hist[b--];
                sh.bin = b;
                sh.above = above;
            }
            __syncthreads();
            thr |= (uint64_t)sh.bin << sh_bits;
            need -= sh.above;
            if (k - need + sh.hist[sh.bin] <= kTopCand) break;
        }
        __syncthreads();
        if (tid == 0) sh.n = 0;
        __syncthreads();
        rest = 0.f;
        each_piece<NT, 4>(row, tid, V, [&](u32x4 w, int i) {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                if (i * N + e >= V) continue;
                const float v = Piece<L>::get(w, e);
                const uint64_t key = pair_key(value_key(v), i * N + e);
                if (key >= thr) sh.cand[atomicAdd(&sh.n, 1)] = key;
                else rest += term(v);
            }
        });
        __syncthreads();
        nc = sh.n;
    }
    // ranked by counting the larger ones
    for (int i = tid; i < nc; i += NT) {
        const uint64_t key = sh.cand[i];
        int rank = 0;
        for (int j = 0; j < nc; ++j) rank += sh.cand[j] > key;
        sh.sorted[rank] = key;
    }
    __syncthreads();
    for (int j = k + tid; j < nc; j += NT) rest += term(key_value((uint32_t)(sh.sorted[j] >> 32)));
    double outside = block_sum<NT>(rest, sh.red[2]);
    if (wave != 0) return;
    // in multiples of exp(max / temperature)
    if (!far && all.m != -INFINITY) outside *= exp((double)B * kLn2 - (double)all.m * p.c.inv);
    double sum = 0.;
    for (int j = lane; j < k; j += 64)
        sum += exp(((double)key_value((uint32_t)(sh.sorted[j] >> 32)) - (double)all.m) * p.c.inv);
    const double lse = log(wave_sum_f64(sum) + outside);    // of x - max / temperature
    for (int j = lane; j < k; j += 64) {
        const uint64_t key = sh.sorted[j];
        p.ids[(int64_t)t * k + j] = key_id(key);
        p.logp[(int64_t)t * k + j] = (float)(((double)key_value((uint32_t)(key >> 32)) - (double)all.m) * p.c.inv - lse);
    }
    if (lane == 0 && p.tail) p.tail[t] = (float)(log(outside) - lse);
}

template <typename L>
static int top_logits(int32_t T, int32_t V, const L *d_logits, int64_t ld, double temperature, int32_t k,
                      int32_t *d_ids, float *d_logp, float *d_tail, void *d_work, int64_t work_bytes, void *stream) {
    (void)d_work; (void)work_bytes;
    if (!opd_rows_ok(T, V, d_logits, ld, temperature, sizeof(L)) || k < 1 || k > kTopMax || k > V) return PIPO_EINVAL;
    if (T == 0) return PIPO_OK;
    if (!d_ids || !d_logp) return PIPO_EINVAL;
    TopParams<L> p{d_logits, ld, T, V, k, exp_scale(temperature), d_ids, d_logp, d_tail};
    if (V > 16384) hipLaunchKernelGGL((k_opd_top<L, 1024>), dim3(T), dim3(1024), 0, (hipStream_t)stream, p);
    else hipLaunchKernelGGL((k_opd_top<L, 256>), dim3(T), dim3(256), 0, (hipStream_t)stream, p);
    return hipGetLastError() == hipSuccess ? PIPO_OK : PIPO_EHIP;
}

}  // namespace pipo

using namespace pipo;

extern "C" int64_t pipo_opd_work_bytes(int32_t T, int32_t V, int32_t k) {
    (void)T; (void)V; (void)k;
    return 0;
}

extern "C" int pipo_opd_top_logits(int32_t T, int32_t V, const float *d_logits, int64_t ld, double temperature,
                                   int32_t k, int32_t *d_ids, float *d_logp, float *d_tail, void *d_work,
                                   int64_t work_bytes, void *stream) {
    return top_logits<float>(T, V, d_logits, ld, temperature, k, d_ids, d_logp, d_tail, d_work, work_bytes, stream);
}

extern "C" int pipo_opd_top_logits_bf16(int32_t T, int32_t V, const uint16_t *d_logits, int64_t ld, double temperature,
                                        int32_t k, int32_t *d_ids, float *d_logp, float *d_tail, void *d_work,
                                        int64_t work_bytes, void *stream) {
    return top_logits<uint16_t>(T, V, d_logits, ld, temperature, k, d_ids, d_logp, d_tail, d_work, work_bytes, stream);
}
