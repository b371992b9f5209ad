// The k largest logits of each row, in the order of (value descending, id
// ascending), with their log-probabilities and the log of the mass outside.
//
// One pass over the row, which is dealt into units of pieces, some to a thread:
// each has its maximum and its sum of exponentials.  A value that at least k
// maxima reach is a lower bound of the k-th largest logit, so only those units
// can hold the k largest: they are read again (about k of 1024, from the
// caches), and what reaches the bound, usually little more than k values, is
// ranked by counting.  Units that hold none of the k keep their sums; the
// others' are added up again without them, so that the mass outside
// the list is a sum of what is outside, not a difference.
// Rows whose values crowd at the bound (constant rows, long ties) overflow the
// candidate array; a radix select over (value, id) keys, which are all
// different, then narrows the row to what fits.
// Where there are too few rows for the chip, each is split over several
// workgroups, and a last one picks the row's k among the segments' lists.
// HBM-bound: V logits read per row.  Top 32 of 2048 x 151936: bf16 120 us, 5.2
// TB/s, fp32 221 us, 5.6 TB/s; what a row adds to its stream (the barriers, the
// search, the units read again) is hidden as far as four workgroups a compute
// unit overlap.
#include "opd_rows.h"
#include "pipo.h"

namespace pipo {

constexpr int kTopMax = 256;        // k
constexpr int kTopCand = 1024;      // candidates ranked
constexpr int kJoinThreads = 1024;

template <typename L> struct TopParams {
    const L *z; int64_t ld;
    int T, V, k;
    ExpScale c;
    int32_t *ids; float *logp, *tail;
    // of a split row: S segments of seg elements, each with a sorted list of k keys (0: none) and its other values' sum
    int S, seg;
    Part *part;                     // [T][S]
    uint64_t *keys;                 // [T][S][k]
};

// Unsigned integers in the order of the values; -0 counts as 0.  0 stands for no
// value: the NaN of all ones, which would have it, shares the next NaN's.
__device__ __forceinline__ uint32_t value_key(float v) {
    const uint32_t u = __float_as_uint(v + 0.f);
    return max((u & 0x80000000u) ? ~u : u | 0x80000000u, 1u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
    return __uint_as_float((k & 0x80000000u) ? k & 0x7FFFFFFFu : ~k);
}
// (value, id) keys: all different, larger for larger values and then for lower ids.
__device__ __forceinline__ uint64_t pair_key(uint32_t vkey, int id) {
    return ((uint64_t)vkey << 32) | (uint32_t)~(uint32_t)id;
}
__device__ __forceinline__ int key_id(uint64_t k) { return (int)~(uint32_t)k; }

template <int NT, int H> struct TopShared {
    uint32_t umax[NT * H];          // each unit's largest value key, 0: no pieces
    uint64_t cand[kTopCand];
    uint64_t sorted[kTopCand];
    Reduce<NT> red;
    uint32_t wmin[NT / 64];
    int count[2][NT / 64], wcount[NT / 64];
    int hist[256];
    int n, bin, above;
};

// A bound that at least k of the keys in sh.umax reach, and few more: each round every
// wave counts the keys at or above a pivot of its own, so a round cuts the range
// by the number of waves plus one.  lo is reached by at least k, none is above hi.
template <int NT, int H>
__device__ __forceinline__ uint32_t bound_of_kth(TopShared<NT, H> &sh, uint32_t lo, uint32_t hi, int k) {
    constexpr int W = NT / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t key[W * H];
#pragma unroll
    for (int i = 0; i < W * H; ++i) key[i] = sh.umax[i * 64 + lane];
    for (int round = 0; lo < hi; ++round) {
        const uint64_t span = (uint64_t)(hi - lo) + 1;
        const uint32_t pivot = lo + (uint32_t)(span * (wave + 1) / (W + 1));
        int n = 0;
#pragma unroll
        for (int i = 0; i < W * H; ++i) n += __popcll(__ballot(key[i] >= pivot));
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

// Sorts sh.cand[0, nc) into sh.sorted: each ranked by counting the larger ones,
// where there are many by several threads each.
template <int NT, int H> __device__ __forceinline__ void sort_candidates(TopShared<NT, H> &sh, int nc) {
    if (nc > 64 && 2 * nc <= NT) {
        int *ranks = (int *)sh.umax;            // (whose keys nobody reads any more)
        const int share = NT / nc, len = (nc + share - 1) / share;
        for (int i = threadIdx.x; i < nc; i += NT) ranks[i] = 0;
        __syncthreads();
        if ((int)threadIdx.x < nc * share) {
            const int i = threadIdx.x % nc, from = threadIdx.x / nc * len, to = min(from + len, nc);
            const uint64_t key = sh.cand[i];
            int rank = 0;
#pragma unroll 4
            for (int j = from; j < to; ++j) rank += sh.cand[j] > key;
            atomicAdd(&ranks[i], rank);
        }
        __syncthreads();
        for (int i = threadIdx.x; i < nc; i += NT) sh.sorted[ranks[i]] = sh.cand[i];
    } else {
        for (int i = threadIdx.x; i < nc; i += NT) {
            const uint64_t key = sh.cand[i];
            int rank = 0;
#pragma unroll 8
            for (int j = 0; j < nc; ++j) rank += sh.cand[j] > key;
            sh.sorted[rank] = key;
        }
    }
    __syncthreads();
}
// The row's outputs, by its first wave: sorted[0, k) are the k largest, m the largest, `out` the sum of all others.
template <typename L>
__device__ __forceinline__ void put_top(const TopParams<L> &p, int t, const uint64_t *sorted, float m, RowSum out) {
    const int lane = threadIdx.x;
    const bool none = out.m == -INFINITY;
    const double unit = none ? 0. : log_unit(out.m, out.B, m, p.c), mass = out.s * exp(unit);
    double sum = 0.;
    for (int j = lane; j < p.k; j += 64)
        sum += exp(((double)key_value((uint32_t)(sorted[j] >> 32)) - (double)m) * p.c.inv);
    const double lse = log(wave_sum_f64(sum) + mass);   // of x - m / temperature
    for (int j = lane; j < p.k; j += 64) {
        const uint64_t key = sorted[j];
        p.ids[(int64_t)t * p.k + j] = key_id(key);
        p.logp[(int64_t)t * p.k + j] = (float)(((double)key_value((uint32_t)(key >> 32)) - (double)m) * p.c.inv - lse);
    }
    if (lane == 0 && p.tail) p.tail[t] = (float)(log(out.s) + unit - lse);
}
// A sum of exponentials under this share of its reference may have lost some that no float holds (2^-126, of 2^19 at most).
constexpr double kThin = 1e-25;
// The sum of a row's values whose keys are below `last`, over a reference of their own.
template <typename L, int NT>
__device__ __forceinline__ RowSum sum_below(const Span<const L> &row, uint64_t last, ExpScale c, Reduce<NT> &red) {
    constexpr int N = Piece<L>::N;
    float m = -INFINITY, s = 0.f;
    auto below = [&](float v, int i, int e) { return row.has(i, e) && pair_key(value_key(v), row.head + i * N + e) < last; };
    each_piece<NT, 1>(row, (int)threadIdx.x, [&](u32x4 w, int i) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float v = Piece<L>::get(w, e);
            if (below(v, i, e)) m = fmaxf(m, v);
        }
    });
    __syncthreads();
    m = block_max<NT>(m, red.max[0]);
    const bool far = is_far(m, c);
    const float B = ref_of(m, c);
    if (m != -INFINITY) {
        each_piece<NT, 1>(row, (int)threadIdx.x, [&](u32x4 w, int i) {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float v = Piece<L>::get(w, e);
                if (below(v, i, e)) s += far ? exp_diff(v, m, c) : exp_at(v, B, c);
            }
        });
    }
    return RowSum{m, B, block_sum<NT>(s, red.sum[1])};
}

// One workgroup per row, or (SPLIT) per segment of one.
template <typename L, int NT, int H, bool SPLIT>
__global__ __launch_bounds__(NT, 8) void k_opd_top(TopParams<L> p) {
    constexpr int N = Piece<L>::N, W = NT / 64;
    __shared__ TopShared<NT, H> sh;
    const int t = SPLIT ? blockIdx.x / p.S : blockIdx.x, seg = SPLIT ? blockIdx.x % p.S : 0;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int lo = seg * p.seg, V = min(p.seg, p.V - lo), k = min(p.k, V);
    const Span<const L> row(p.z + (int64_t)t * p.ld + lo, V);
    const int n = row.whole;        // (the partial pieces, at most 14 values, are candidates in any case)

    // unit h NT + tid: the pieces tid + NT j for j from h per on, per of them
    const int per = (n + NT * H - 1) / (NT * H);
    MaxSum<float> unit[H];
#pragma unroll
    for (int h = 0; h < H; ++h) {
        unit[h] = MaxSum<float>{-INFINITY, 0.f};
        const int first = tid + h * per * NT, end = (h + 1) * per * NT;
        auto add = [&](u32x4 w, int) {
            float v[N];
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] = Piece<L>::get(w, e);
            add_values<N>(unit[h], v, p.c);
        };
        whole_pieces<NT, 4>(row.body, first, min(end, n), add);
    }
    float least_own = INFINITY, most_own = -INFINITY;
#pragma unroll
    for (int h = 0; h < H; ++h) {
        const bool used = tid + h * per * NT < n;
        sh.umax[h * NT + tid] = used ? value_key(unit[h].m) : 0u;
        if (used) least_own = fminf(least_own, unit[h].m);
        most_own = fmaxf(most_own, unit[h].m);
    }
    edges<NT>(row, [&](u32x4 w, int) {
#pragma unroll
        for (int e = 0; e < N; ++e) most_own = fmaxf(most_own, Piece<L>::get(w, e));
    });
    // the least of them, as the largest of the negated maxima (-0 and 0 have one key)
    const float least_w = -wave_max_dpp(-least_own);
    if (lane == 0) sh.wmin[wave] = value_key(least_w);
    if (tid == 0) sh.n = 0;
    const float m = block_max<NT>(most_own, sh.red.max[0]);     // its barrier: umax, wmin and n are set
    const bool far = is_far(m, p.c);
    const float B = ref_of(m, p.c);
    auto term = [&](float v) { return far ? exp_diff(v, m, p.c) : exp_at(v, B, p.c); };
    uint32_t least = sh.wmin[0];
#pragma unroll
    for (int w = 1; w < W; ++w) least = min(least, sh.wmin[w]);
    // fewer pieces than k: everything is a candidate
    const uint32_t bound = n < k ? 0u : bound_of_kth(sh, least, value_key(m), k);

    // the units that reach the bound, again
    float rest = 0.f;
    uint64_t ball[H];
    int mine = 0;
#pragma unroll
    for (int h = 0; h < H; ++h) {
        const bool used = tid + h * per * NT < n, picked = used && value_key(unit[h].m) >= bound;
        ball[h] = __ballot(picked);
        if (!picked) rest += unit[h].s * __builtin_amdgcn_exp2f(ref_of(unit[h].m, p.c) - B);
        mine += __popcll(ball[h]);
    }
    if (lane == 0) sh.wcount[wave] = mine;
    __syncthreads();                // every wave is past the search: its keys become the picked units
    int at = 0, total = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        const int c = sh.wcount[w];
        if (w < wave) at += c;
        total += c;
    }
    uint32_t *list = sh.umax;
#pragma unroll
    for (int h = 0; h < H; ++h) {
        if (ball[h] >> lane & 1u) list[at + __popcll(ball[h] & ((1ull << lane) - 1))] = h * per * NT + tid;   // its first piece
        at += __popcll(ball[h]);
    }
    __syncthreads();
    auto take = [&](u32x4 w, int i) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float v = Piece<L>::get(w, e);
            const uint32_t key = value_key(v);
            if (key >= bound && row.has(i, e)) {
                const int c = atomicAdd(&sh.n, 1);
                if (c < kTopCand) sh.cand[c] = pair_key(key, row.head + i * N + e);
            } else {
                rest += term(v);
            }
        }
    };
    for (int x0 = tid; x0 < total * per; x0 += 4 * NT) {
        u32x4 w[4];
        int at[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {       // four in flight: this is all latency
            const int x = x0 + u * NT;
            at[u] = x < total * per ? (int)list[x / per] + NT * (x % per) : n;
            if (at[u] < n) w[u] = load_piece(row.body, at[u]);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (at[u] < n) take(w[u], at[u]);
        }
    }
    edges<NT>(row, take);
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
            each_piece<NT, 4>(row, tid, [&](u32x4 w, int i) {
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    if (!row.has(i, e)) continue;
                    const uint64_t key = pair_key(value_key(Piece<L>::get(w, e)), row.head + i * N + e);
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
        each_piece<NT, 4>(row, tid, [&](u32x4 w, int i) {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                if (!row.has(i, e)) continue;
                const float v = Piece<L>::get(w, e);
                const uint64_t key = pair_key(value_key(v), row.head + i * N + e);
                if (key >= thr) sh.cand[atomicAdd(&sh.n, 1)] = key;
                else rest += term(v);
            }
        });
        __syncthreads();
        nc = sh.n;
    }
    sort_candidates(sh, nc);
    for (int j = k + tid; j < nc; j += NT) rest += term(key_value((uint32_t)(sh.sorted[j] >> 32)));
    RowSum out{m, B, block_sum<NT>(rest, sh.red.sum[0])};
    if (out.s < kThin) {
        const uint64_t last = sh.sorted[k - 1];     // (below a last one of -inf, or where all are on the list, there is nothing)
        if (k < V && (uint32_t)(last >> 32) > value_key(-INFINITY)) out = sum_below<L, NT>(row, last, p.c, sh.red);
        else out.m = -INFINITY;
    }
    if (SPLIT) {
        uint64_t *keys = p.keys + ((int64_t)t * p.S + seg) * p.k;
        for (int j = tid; j < p.k; j += NT) {
            const uint64_t key = j < k ? sh.sorted[j] : 0;
            keys[j] = key ? pair_key((uint32_t)(key >> 32), key_id(key) + lo) : 0;
        }
        if (tid == 0) p.part[(int64_t)t * p.S + seg] = Part{out.m, out.B, out.s, 0, 0};
    } else if (wave == 0) {
        put_top(p, t, sh.sorted, m, out);
    }
}

// The k largest of a split row among its segments' lists: S k keys, at most one a thread.
template <typename L> __global__ __launch_bounds__(kJoinThreads) void k_opd_top_join(TopParams<L> p) {
    constexpr int NT = kJoinThreads;
    __shared__ TopShared<NT, 1> sh;
    const int t = blockIdx.x, tid = threadIdx.x, lane = tid & 63, k = p.k;
    const uint64_t *keys = p.keys + (int64_t)t * p.S * k;
    bool bad;
    const RowSum rests = join_parts(p.part + (int64_t)t * p.S, p.S, p.c, bad);
    const uint64_t mine = tid < p.S * k ? keys[tid] : 0;
    // a whole list reaches its own last key: the largest of these is a bound that k keys reach
    uint32_t lo = lane < p.S ? (uint32_t)(keys[(int64_t)lane * k + k - 1] >> 32) : 0;
    uint32_t hi = lane < p.S ? (uint32_t)(keys[(int64_t)lane * k] >> 32) : 0;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        lo = max(lo, (uint32_t)__shfl_xor((int)lo, o));
        hi = max(hi, (uint32_t)__shfl_xor((int)hi, o));
    }
    lo = max(lo, 1u);
    sh.umax[tid] = (uint32_t)(mine >> 32);
    if (tid == 0) sh.n = 0;
    __syncthreads();
    const uint32_t bound = bound_of_kth(sh, lo, hi, k);
    if (mine && (uint32_t)(mine >> 32) >= bound) sh.cand[atomicAdd(&sh.n, 1)] = mine;
    __syncthreads();
    sort_candidates(sh, sh.n);
    // the lists' other keys and the segments' other values, over the row's largest value, or where that is thin over their own
    const float top = key_value((uint32_t)(sh.sorted[0] >> 32)), v = key_value((uint32_t)(mine >> 32));
    const bool other = mine && mine < sh.sorted[k - 1];
    auto sum_over = [&](float m, double *s_w) {
        const bool far = is_far(m, p.c);
        const float B = ref_of(m, p.c), term = !other ? 0.f : far ? exp_diff(v, m, p.c) : exp_at(v, B, p.c);
        double f = 1.;      // the segments' unit over this one: as a rule the same
        if (rests.m != m && rests.m != -INFINITY) f = exp(log_unit(rests.m, rests.B, m, p.c) - (far ? 0. : log_unit(m, B, m, p.c)));
        return RowSum{m, B, block_sum<NT>(term, s_w) + rests.s * f};
    };
    RowSum out = sum_over(top, sh.red.sum[0]);
    if (out.s < kThin) out = sum_over(fmaxf(block_max<NT>(other ? v : -INFINITY, sh.red.max[0]), rests.m), sh.red.sum[1]);
    if (tid < 64) put_top(p, t, sh.sorted, top, out);
}

// Segments of each row: about two workgroups a compute unit in all, at least
// 4096 elements each, and no more keys than the joining workgroup has threads.
// Two launches pay for few long rows (bf16, top 20, us for split / whole): 8 x
// 65536 16.7 / 13.0, 8 x 151936 17.0 / 21.1, 64 x 151936 19.8 / 23.0, 128 x
// 151936 24.1 / 23.7.
static void top_split(int T, int V, int k, int es, int &S, int &seg) {
    S = 512 / T;
    if (S > kMaxParts) S = kMaxParts;
    if (S > V / 4096) S = V / 4096;
    if (S > kJoinThreads / k) S = kJoinThreads / k;
    if (S < 2 || T > 96 || (int64_t)V * es < 256 << 10) { S = 1; seg = V; return; }
    seg = ((V + S - 1) / S + 255) / 256 * 256;
    S = (V + seg - 1) / seg;
}
static int64_t top_bytes(int T, int V, int k, int es) {
    int S, seg;
    top_split(T, V, k, es, S, seg);
    return S > 1 ? (int64_t)T * S * ((int64_t)sizeof(Part) + (int64_t)k * 8) : 0;
}

template <typename L>
static int top_logits(int32_t T, int32_t V, const L *d_logits, int64_t ld, double temperature, int32_t k,
                      int32_t *d_ids, float *d_logp, float *d_tail, void *d_work, int64_t work_bytes, void *stream) {
    if (!opd_rows_ok(T, V, d_logits, ld, temperature, sizeof(L)) || k < 1 || k > kTopMax || k > V) return PIPO_EINVAL;
    if (T == 0) return PIPO_OK;
    if (!d_ids || !d_logp || !opd_work_ok(d_work, work_bytes, top_bytes(T, V, k, sizeof(L)))) return PIPO_EINVAL;
    TopParams<L> p{d_logits, ld, T, V, k, exp_scale(temperature), d_ids, d_logp, d_tail, 1, V, nullptr, nullptr};
    hipStream_t s = (hipStream_t)stream;
    if (d_work && top_bytes(T, V, k, sizeof(L)) > 0) {
        top_split(T, V, k, sizeof(L), p.S, p.seg);
        p.part = (Part *)d_work;
        p.keys = (uint64_t *)(p.part + (int64_t)T * p.S);
        return launch(k_opd_top<L, 256, 2, true>, T * p.S, 256, 0, s, p) && launch(k_opd_top_join<L>, T, kJoinThreads, 0, s, p)
                   ? PIPO_OK : PIPO_EHIP;
    }
    // Threads and units a thread: enough units to leave little to read again, few to search.  Two / four units, us:
    // 2048 x 151936 fp32 240 / 221, 2048 x 100003 fp32 top 100 213 / 184, 301 x 151936 bf16 33 / 36; one / two: 16384 x
    // 4096 fp32 86 / 105, 4000 x 12003 fp32 91 / 74.
    const int pieces = V / (16 / (int)sizeof(L));
    const bool ok = pieces >= 20480 ? launch(k_opd_top<L, 512, 4, false>, T, 512, 0, s, p)
                    : V > 16384      ? launch(k_opd_top<L, 512, 2, false>, T, 512, 0, s, p)
                    : pieces <= 1024 ? launch(k_opd_top<L, 256, 1, false>, T, 256, 0, s, p)
                                     : launch(k_opd_top<L, 256, 2, false>, T, 256, 0, s, p);
    return ok ? PIPO_OK : PIPO_EHIP;
}

}  // namespace pipo

using namespace pipo;

extern "C" int64_t pipo_opd_work_bytes(int32_t call, int32_t T, int32_t V, int32_t k, int32_t bf16) {
    const int es = bf16 ? 2 : 4;
    if (T < 1 || V < 1 || V > kOpdMaxVocab || k < 1 || k > kTopMax) return 0;
    return call == PIPO_OPD_CALL_TOP ? top_bytes(T, V, k, es) : opd_loss_work_bytes(T, V, k, es, call == PIPO_OPD_CALL_GRAD);
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
