// Grouped-query attention of a step's tokens over the paged 8-bit cache.
//
// A unit is up to 16 NCT query rows (tokens x the group's heads) of one request and KV head
// and a range of 32-token tiles.  Scores are computed transposed, S^T[token][row] =
// K Q^T, so that a lane's accumulators belong to one row, and the probabilities
// are already the B operand of O^T[dim][row] += V^T P^T in the value tiles' token
// order.  The bytes become fp16 exactly (1024 + u by a byte permutation, less
// 1152), the scales go into the scores and into what each tile adds to O.  Queries
// are brought to magnitudes below 2^15 by a power of two for each row, and probabilities are
// kept as 2^14 times themselves, so that fp16's exponents hold them; bf16 queries
// are then fp16 numbers (parts below 2^-38 of the row's largest are lost), and probabilities
// lose 2^-12 of themselves, an eighth of what the output's rounding to bf16 costs.  fp32
// queries, and their probabilities, go in as hi + lo fp16 pairs (2^-22), two MFMAs each.
#include "kv8.h"
#include <math.h>

namespace pipo {

struct Kv8Attn {
    const uint8_t *keys, *values;
    const float *scales;
    const int32_t *tables, *starts, *total;
    const void *q; void *out;
    int64_t ld_q, ld_out;
    int R, rows, W, blocks, n_kv, n_q, qpg, shift, max_len;     // block = 1 << shift
    int S, chunk;                   // key ranges of `chunk` tiles
    int groups;                     // row groups of all requests, counted from above
    float scale;                    // of the scores, times log2(e)
    float *part;                    // [groups][n_kv][S][16 NCT][D + 2]
};

__device__ __forceinline__ f32x4 mfma16_f16(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
// Eight bytes u as fp16 u - 128: 0x6400 | u is 1024 + u.
__device__ __forceinline__ u32x4 widen8(uint32_t a, uint32_t b) {
    const f16x2_t off = {(_Float16)1152.f, (_Float16)1152.f};
    const uint32_t w[4] = {__builtin_amdgcn_perm(0x64646464u, a, 0x04010400u), __builtin_amdgcn_perm(0x64646464u, a, 0x04030402u),
                           __builtin_amdgcn_perm(0x64646464u, b, 0x04010400u), __builtin_amdgcn_perm(0x64646464u, b, 0x04030402u)};
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2_t, w[i]) - off);
    return r;
}
__device__ __forceinline__ float f16_lo(uint32_t w) { return (float)__builtin_bit_cast(f16x2_t, w)[0]; }
__device__ __forceinline__ float f16_hi(uint32_t w) { return (float)__builtin_bit_cast(f16x2_t, w)[1]; }
template <bool PAIR> __device__ __forceinline__ void fp16_8(const float *v, u32x4 &hi, u32x4 &lo) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        hi[i] = pack_f16x2(v[2 * i], v[2 * i + 1]);
        if (PAIR) lo[i] = pack_f16x2(v[2 * i] - f16_lo(hi[i]), v[2 * i + 1] - f16_hi(hi[i]));
    }
}

// Where a row group lies: request r's groups are numbered from start(r) * qpg / (16 NCT) + r
// on, which leaves room for the part-filled last one of every request before it.
struct RowGroup { int r, row0, n, first, last; };   // rows row0 .. of the request's n * qpg; last: its total, cut off
template <int ROWS> __device__ __forceinline__ bool find_group(const Kv8Attn &p, int f, RowGroup &g) {
    auto at = [&](int r) { return (int)(((int64_t)max(p.starts[r], 0) * p.qpg) / ROWS) + r; };
    int lo = 0, hi = p.R;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (at(mid) <= f) lo = mid; else hi = mid;
    }
    g.r = lo;
    g.first = max(p.starts[lo], 0);
    g.n = min(p.starts[lo + 1], p.rows) - g.first;
    g.row0 = (f - at(lo)) * ROWS;
    g.last = min(max(p.total[lo], 0), p.max_len);
    return g.row0 >= 0 && g.row0 < g.n * p.qpg;
}
// Tiles that the rows of a group see: up to its last token's position.
template <int ROWS> __device__ __forceinline__ int tiles_of(const Kv8Attn &p, const RowGroup &g, int total) {
    const int i = min(g.row0 + ROWS, g.n * p.qpg) - 1, seen = min(total - g.n + i / p.qpg + 1, g.last);
    return seen > 0 ? (seen + 31) >> 5 : 0;
}

// The four waves of a workgroup share a row group and cut its key range into four
// (SPLIT), or take a row group each.
template <typename L, int D, int NCT, bool SPLIT>
__global__ __launch_bounds__(256, (NCT > 2 || (NCT > 1 && sizeof(L) == 4)) ? 1 : 2) void k_kv8_attn(Kv8Attn p) {
    constexpr bool PAIR = sizeof(L) == 4;
    constexpr int ROWS = 16 * NCT, NC = D / 64, NT = D / 16, NV = D / 32;
    const int lane = threadIdx.x & 63, j = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    int x = blockIdx.x;
    const int head = x % p.n_kv;
    x /= p.n_kv;
    const int split = x % p.S, f = x / p.S * (SPLIT ? 1 : 4) + (SPLIT ? 0 : wave);
    RowGroup rg;
    bool live = f < p.groups && find_group<ROWS>(p, f, rg);
    if (!live) {
        if (SPLIT) return;
        rg = RowGroup{0, 0, 0, 0, 0};
    }
    const int total = live ? p.total[rg.r] : 0;
    const int tiles = live ? tiles_of<ROWS>(p, rg, total) : 0;
    const int t_lo = split * p.chunk, t_hi = min(t_lo + p.chunk, tiles);
    if (SPLIT ? t_lo >= t_hi && split > 0 : false) return;
    if (!SPLIT && (!live || (t_lo >= t_hi && split > 0))) return;
    const int n_split = tiles > 0 ? (tiles + p.chunk - 1) / p.chunk : 1;
    int ta = t_lo, tb = max(t_hi, t_lo);
    if (SPLIT) {
        const int n = tb - t_lo;
        ta = t_lo + (n * wave >> 2);
        tb = t_lo + (n * (wave + 1) >> 2);
    }
    // this lane's query rows
    u32x4 qh[NCT][NC][2], ql[NCT][NC][2];
    float fq[NCT];                  // the row's factor of the scores
    int seen[NCT], row_at[NCT], head_at[NCT];   // tokens it sees; its output row (-1: none) and head
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct) {
        const int rr = rg.row0 + 16 * ct + j, i = rr / p.qpg, h = head * p.qpg + rr - i * p.qpg;
        const bool is = i < rg.n;
        row_at[ct] = is ? rg.first + i : -1;
        head_at[ct] = h;
        seen[ct] = is ? max(min(total - rg.n + i + 1, rg.last), 0) : 0x7FFFFFFF;    // (what is no row is not written)
        float v[NC][16];
        const L *q = (const L *)p.q + (is ? row_at[ct] * p.ld_q + (int64_t)h * D + 16 * g : 0);
        float top = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int e = 0; e < 16; e += Piece<L>::N) {
                u32x4 w{0u, 0u, 0u, 0u};
                if (is) w = *(const typename Piece<L>::raw_t *)(q + 64 * c + e);
#pragma unroll
                for (int k = 0; k < Piece<L>::N; ++k) {
                    v[c][e + k] = Piece<L>::get(w, k);
                    top = fmaxf(top, fabsf(v[c][e + k]));
                }
            }
        top = col_max(top);
        // the power of two that brings the largest to [2^14, 2^15)
        const int ex = top > 0.f && top < INFINITY ? 14 - ilogbf(top) : 0;
        fq[ct] = ldexpf(p.scale, -ex);
#pragma unroll
        for (int c = 0; c < NC; ++c) {
#pragma unroll
            for (int e = 0; e < 16; ++e) v[c][e] = ldexpf(v[c][e], ex);
            fp16_8<PAIR>(v[c], qh[ct][c][0], ql[ct][c][0]);
            fp16_8<PAIR>(v[c] + 8, qh[ct][c][1], ql[ct][c][1]);
        }
    }
    int all_see = 0x7FFFFFFF;       // tokens that every row sees
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct) all_see = min(all_see, seen[ct]);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) all_see = min(all_see, __shfl_xor(all_see, o));
    all_see = __builtin_amdgcn_readfirstlane(all_see);

    f32x4 o[NCT][NT];
    float m_run[NCT], l_run[NCT];
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct) {
        m_run[ct] = -INFINITY;
        l_run[ct] = 0.f;
#pragma unroll
        for (int t = 0; t < NT; ++t) o[ct][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // A lane holds the number and scales of one of 64 blocks from blk0 on.
    const int sh = p.shift - 5;     // tiles of a block: 1 << sh
    int blk0 = 0, id = -1;
    float2 sc = make_float2(0.f, 0.f);
    auto load_ids = [&](int b0) {
        blk0 = b0;
        const int at = b0 + lane;
        id = at < p.W ? p.tables[(int64_t)rg.r * p.W + at] : -1;
        if ((unsigned)id >= (unsigned)p.blocks) id = -1;
        sc = id >= 0 ? *(const float2 *)(p.scales + ((int64_t)id * p.n_kv + head) * 2) : make_float2(0.f, 0.f);
    };
    u32x4 kf[2][2][NC], vf[2][NV];
    int at_id[2];
    float at_k[2], at_v[2];
    auto load_tile = [&](int buf, int t) {
        const int tc = min(t, tb - 1), b = tc >> sh;
        if (b - blk0 >= 64) load_ids(b);
        const int bi = b - blk0, bid = __builtin_amdgcn_readlane(id, bi);
        at_id[buf] = bid;
        at_k[buf] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(sc.x), bi));
        at_v[buf] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(sc.y), bi));
        const int64_t off = ((((int64_t)max(bid, 0) * p.n_kv + head) << p.shift) + ((tc & ((1 << sh) - 1)) << 5)) * D;
        const u32x4 *k = (const u32x4 *)(p.keys + off) + lane, *v = (const u32x4 *)(p.values + off) + lane;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int c = 0; c < NC; ++c) kf[buf][u][c] = SPLIT ? __builtin_nontemporal_load(k + (u * NC + c) * 64) : k[(u * NC + c) * 64];
#pragma unroll
        for (int c = 0; c < NV; ++c) vf[buf][c] = SPLIT ? __builtin_nontemporal_load(v + c * 64) : v[c * 64];
    };
    auto tile = [&](int buf, int t) {
        if (at_id[buf] < 0) return;         // no such block: its tokens are not there
        f32x4 st[NCT][2];
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
            for (int u = 0; u < 2; ++u) st[ct][u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const u32x4 a = widen8(kf[buf][u][c][2 * e], kf[buf][u][c][2 * e + 1]);
#pragma unroll
                    for (int ct = 0; ct < NCT; ++ct) {
                        st[ct][u] = mfma16_f16(a, qh[ct][c][e], st[ct][u]);
                        if (PAIR) st[ct][u] = mfma16_f16(a, ql[ct][c][e], st[ct][u]);
                    }
                }
        const int t0 = t * 32;
        const bool whole = t0 + 32 <= all_see;
        u32x4 ph[NCT], pl[NCT];
        float al[NCT], sv[NCT];
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct) {
            const float fk = fq[ct] * at_k[buf];
            float mx = -INFINITY, pf[8];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    float s = st[ct][u][v] * fk;
                    if (!whole && t0 + 16 * u + 4 * g + v >= seen[ct]) s = -INFINITY;
                    pf[4 * u + v] = s;
                    mx = fmaxf(mx, s);
                }
            const float m_new = fmaxf(m_run[ct], col_max(mx));
            const float ref = m_new == -INFINITY ? 0.f : m_new;
            al[ct] = __builtin_amdgcn_exp2f(m_run[ct] - ref);
            m_run[ct] = m_new;
            float sum = 0.f;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                pf[k] = __builtin_amdgcn_exp2f(pf[k] - ref + 14.f);
                sum += pf[k];
            }
            l_run[ct] = l_run[ct] * al[ct] + sum;
            fp16_8<PAIR>(pf, ph[ct], pl[ct]);
            sv[ct] = t0 < seen[ct] ? at_v[buf] : 0.f;   // (a row that sees nothing of the tile gets nothing of its scale)
        }
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const u32x4 a = widen8(vf[buf][c][2 * e], vf[buf][c][2 * e + 1]);
#pragma unroll
                for (int ct = 0; ct < NCT; ++ct) {
                    f32x4 w = mfma16_f16(a, ph[ct], f32x4{0.f, 0.f, 0.f, 0.f});
                    if (PAIR) w = mfma16_f16(a, pl[ct], w);
#pragma unroll
                    for (int v = 0; v < 4; ++v) o[ct][2 * c + e][v] = fmaf(w[v], sv[ct], o[ct][2 * c + e][v] * al[ct]);
                }
            }
    };
    if (ta < tb) {
        load_ids(ta >> sh);
        load_tile(0, ta);
        load_tile(1, ta + 1);
        int t = ta;
        for (; t + 2 < tb; t += 2) {
            tile(0, t);
            load_tile(0, t + 2);
            tile(1, t + 1);
            load_tile(1, t + 3);
        }
        tile(0, t);
        if (t + 1 < tb) tile(1, t + 1);
    }
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct) l_run[ct] = col_sum(l_run[ct]);

    // to the output, or as a record for the others of the row's key ranges
    auto finish = [&](int ct, int rr, int row, int h, int d, float a, float b, float c, float e, float m, float l, bool stat) {
        if (row < 0) return;
        if (n_split == 1) {
            const float inv = l == 0.f ? 0.f : 1.f / l;
            L *to = (L *)p.out + row * p.ld_out + (int64_t)h * D + d;
            Piece<L>::put(to, a * inv);
            Piece<L>::put(to + 1, b * inv);
            Piece<L>::put(to + 2, c * inv);
            Piece<L>::put(to + 3, e * inv);
        } else {
            float *rec = p.part + ((((int64_t)f * p.n_kv + head) * p.S + split) * ROWS + 16 * ct + rr) * (D + 2);
            *(float2 *)(rec + d) = make_float2(a, b);
            *(float2 *)(rec + d + 2) = make_float2(c, e);
            if (stat) *(float2 *)(rec + D) = make_float2(m, l);
        }
    };
    if constexpr (!SPLIT) {
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
            for (int t = 0; t < NT; ++t)
                finish(ct, j, row_at[ct], head_at[ct], 16 * t + 4 * g, o[ct][t][0], o[ct][t][1], o[ct][t][2], o[ct][t][3],
                       m_run[ct], l_run[ct], t == 0 && g == 0);
    } else {
        __shared__ float red[4][16][D + 2];
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct) {
            if (ct > 0) __syncthreads();
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int v = 0; v < 4; v += 2)
                    *(float2 *)&red[wave][j][16 * t + 4 * g + v] = make_float2(o[ct][t][v], o[ct][t][v + 1]);
            if (g == 0) *(float2 *)&red[wave][j][D] = make_float2(m_run[ct], l_run[ct]);
            __syncthreads();
            for (int e = threadIdx.x; e < 16 * D / 4; e += 256) {
                const int rr = e / (D / 4), d = e % (D / 4) * 4, at = rg.row0 + 16 * ct + rr, i = at / p.qpg;
                if (i >= rg.n) continue;
                float M = -INFINITY, l = 0.f, a[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < 4; ++w) M = fmaxf(M, red[w][rr][D]);
                const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const float k = __builtin_amdgcn_exp2f(red[w][rr][D] - ref);
                    l += k * red[w][rr][D + 1];
#pragma unroll
                    for (int v = 0; v < 4; ++v) a[v] += k * red[w][rr][d + v];
                }
                finish(ct, rr, rg.first + i, head * p.qpg + at - i * p.qpg, d, a[0], a[1], a[2], a[3], M, l, d == 0);
            }
        }
    }
}

// The key ranges' records of a row as one: a wave a row, D / 64 dimensions a lane.
template <typename L, int D, int NCT> __global__ __launch_bounds__(256) void k_kv8_attn_join(Kv8Attn p) {
    constexpr int ROWS = 16 * NCT, E = D / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int head = blockIdx.x % p.n_kv, f = blockIdx.x / p.n_kv;
    RowGroup rg;
    if (!find_group<ROWS>(p, f, rg)) return;
    const int tiles = tiles_of<ROWS>(p, rg, p.total[rg.r]);
    const int n = (tiles + p.chunk - 1) / p.chunk;
    if (n <= 1) return;             // the unit wrote it out itself
    for (int rr = wave; rr < ROWS && rg.row0 + rr < rg.n * p.qpg; rr += 4) {
        const float *rec = p.part + (((int64_t)f * p.n_kv + head) * p.S * ROWS + rr) * (D + 2);
        const int64_t step = (int64_t)ROWS * (D + 2);
        float M = -INFINITY, l = 0.f, a[E];
#pragma unroll
        for (int e = 0; e < E; ++e) a[e] = 0.f;
        for (int s = 0; s < n; ++s) M = fmaxf(M, rec[s * step + D]);
        const float ref = M == -INFINITY ? 0.f : M;
        for (int s = 0; s < n; ++s) {
            const float k = __builtin_amdgcn_exp2f(rec[s * step + D] - ref);
            l += k * rec[s * step + D + 1];
#pragma unroll
            for (int e = 0; e < E; ++e) a[e] += k * rec[s * step + lane * E + e];
        }
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const int i = (rg.row0 + rr) / p.qpg, h = head * p.qpg + rg.row0 + rr - i * p.qpg;
        L *to = (L *)p.out + (rg.first + i) * p.ld_out + (int64_t)h * D + lane * E;
#pragma unroll
        for (int e = 0; e < E; ++e) Piece<L>::put(to + e, a[e] * inv);
    }
}

// ---- shapes of a launch ----------------------------------------------------------------
struct Kv8Shape { int nct, S, chunk, groups; bool split; int64_t part; };
static Kv8Shape shape_of(int R, int rows, int n_q, int n_kv, int D, int max_len, int es, bool work) {
    Kv8Shape s{};
    const int qpg = n_q / n_kv, most = es == 4 ? 2 : 4;
    const int64_t per = ((int64_t)(rows + R - 1) / R) * qpg;        // query rows of a request and KV head, on average
    s.nct = per <= 16 ? 1 : per <= 32 || most == 2 ? 2 : 4;
    const int64_t tile_rows = 16 * s.nct;
    s.groups = (int)((int64_t)rows * qpg / tile_rows) + R;
    const int64_t units = (int64_t)R * ((per + tile_rows - 1) / tile_rows) * n_kv;
    const int tiles = (max_len + 31) / 32;
    s.split = s.nct < most || units < 1024;
    s.S = 1;
    if (work && s.split && units < 1024) {
        int64_t S = (1024 + units - 1) / units;
        if (S > tiles / 8) S = tiles / 8;
        s.S = S < 1 ? 1 : (int)S;
    }
    s.chunk = (tiles + s.S - 1) / s.S;
    s.S = (tiles + s.chunk - 1) / s.chunk;
    s.part = s.S > 1 ? (int64_t)s.groups * n_kv * s.S * tile_rows * (D + 2) * 4 : 0;
    return s;
}

template <typename L, int D, int NCT, bool SPLIT> static bool run_attn(const Kv8Attn &p, hipStream_t s) {
    const int64_t grid = (int64_t)(SPLIT ? p.groups : (p.groups + 3) / 4) * p.S * p.n_kv;
    if (!launch(k_kv8_attn<L, D, NCT, SPLIT>, (unsigned)grid, 256, 0, s, p)) return false;
    return p.S == 1 || launch(k_kv8_attn_join<L, D, NCT>, (unsigned)(p.groups * p.n_kv), 256, 0, s, p);
}
template <typename L, int D> static bool run_attn_d(const Kv8Attn &p, const Kv8Shape &s, hipStream_t st) {
    constexpr int most = sizeof(L) == 4 ? 2 : 4;
    if (s.nct == 1) return run_attn<L, D, 1, true>(p, st);
    if (most == 4 && s.nct == 2) return run_attn<L, D, 2, true>(p, st);
    return s.split ? run_attn<L, D, most, true>(p, st) : run_attn<L, D, most, false>(p, st);
}

static bool attn_sizes_ok(const pipo_kv8 *c, int32_t R, int32_t rows, int32_t n_q, int32_t max_len) {
    return kv8_ok(c) && R >= 1 && R <= kKv8MaxRows && rows >= 0 && rows <= kKv8MaxRows && n_q >= 1 && n_q % c->n_kv == 0 &&
           n_q / c->n_kv <= 16 && max_len >= 1 &&
           ((int64_t)rows * (n_q / c->n_kv) / 16 + R) * c->n_kv < (int64_t)1 << 24;
}

template <typename L>
static int attention(const pipo_kv8 *c, int32_t R, int32_t rows, int32_t n_q, const L *q, int64_t ld_q,
                     const int32_t *tables, int32_t width, const int32_t *starts, const int32_t *total, int32_t max_len,
                     double scale, L *out, int64_t ld_out, void *work, int64_t work_bytes, void *stream) {
    if (!attn_sizes_ok(c, R, rows, n_q, max_len) || width < 1 || max_len > (int64_t)width * c->block || !isfinite((float)scale))
        return PIPO_EINVAL;
    if (rows == 0) return PIPO_OK;
    const int64_t least = (int64_t)n_q * c->head_dim;
    if (!kv8_aligned(q, sizeof(L)) || !kv8_aligned(out, sizeof(L)) || !kv8_aligned(tables, 4) || !kv8_aligned(starts, 4) ||
        !kv8_aligned(total, 4))
        return PIPO_EINVAL;
    if (rows > 1 && (ld_q < least || ld_out < least || ld_q > (int64_t)1 << 31 || ld_out > (int64_t)1 << 31)) return PIPO_EINVAL;
    const Kv8Shape s = shape_of(R, rows, n_q, c->n_kv, c->head_dim, max_len, sizeof(L), work != nullptr);
    if (work && s.part > 0 && (!kv8_aligned(work, 16) || work_bytes < s.part)) return PIPO_EINVAL;
    Kv8Attn p{c->keys, c->values, c->scales, tables, starts, total, q, out, ld_q, ld_out, R, rows, width, c->blocks,
              c->n_kv, n_q, n_q / c->n_kv, __builtin_ctz((unsigned)c->block), max_len, s.S, s.chunk, s.groups,
              (float)(scale * 1.4426950408889634074), (float *)work};
    hipStream_t st = (hipStream_t)stream;
    return (c->head_dim == 128 ? run_attn_d<L, 128>(p, s, st) : run_attn_d<L, 64>(p, s, st)) ? PIPO_OK : PIPO_EHIP;
}

}  // namespace pipo

using namespace pipo;

extern "C" int64_t pipo_kv8_attention_work_bytes(const pipo_kv8 *c, int32_t R, int32_t rows, int32_t n_q, int32_t max_len,
                                                 int32_t bf16) {
    if (!attn_sizes_ok(c, R, rows, n_q, max_len) || rows == 0) return 0;
    return shape_of(R, rows, n_q, c->n_kv, c->head_dim, max_len, bf16 ? 2 : 4, true).part;
}

extern "C" int pipo_kv8_attention(const pipo_kv8 *cache, int32_t R, int32_t rows, int32_t n_q, const float *d_q,
                                  int64_t ld_q, const int32_t *d_tables, int32_t width, const int32_t *d_starts,
                                  const int32_t *d_total, int32_t max_len, double scale, float *d_out, int64_t ld_out,
                                  void *d_work, int64_t work_bytes, void *stream) {
    return attention<float>(cache, R, rows, n_q, d_q, ld_q, d_tables, width, d_starts, d_total, max_len, scale, d_out,
                            ld_out, d_work, work_bytes, stream);
}
extern "C" int pipo_kv8_attention_bf16(const pipo_kv8 *cache, int32_t R, int32_t rows, int32_t n_q, const uint16_t *d_q,
                                       int64_t ld_q, const int32_t *d_tables, int32_t width, const int32_t *d_starts,
                                       const int32_t *d_total, int32_t max_len, double scale, uint16_t *d_out,
                                       int64_t ld_out, void *d_work, int64_t work_bytes, void *stream) {
    return attention<uint16_t>(cache, R, rows, n_q, d_q, ld_q, d_tables, width, d_starts, d_total, max_len, scale, d_out,
                               ld_out, d_work, work_bytes, stream);
}
