// Grouped-query attention of a step's tokens over the paged 8-bit cache.
//
// A unit is up to 16 NCT query rows (tokens x the group's heads) of one request and KV head
// and a range of 32-token tiles.  Scores are computed transposed, S^T[token][row] =
// K Q^T, so that a lane's accumulators belong to one row, and the probabilities
// are already the B operand of O^T[dim][row] += V^T P^T in the value tiles' token
// order.  Value bytes become fp16 exactly (1024 + u by a byte permutation, less
// 1152); key bytes go in as fp16's smallest numbers, u 2^-24, for bf16 queries, whose
// scores are then less 128 times the query's sum, and like the values for fp32 ones.
// Scales go into the scores and into the probabilities (fp32: into what a tile adds to
// O).  Queries are brought to magnitudes below 2^15 by a power of two for each row, and
// probabilities are kept as a power of two times themselves, so that fp16's exponents hold
// them: bf16 queries are then fp16 numbers (parts below 2^-38 of the row's largest are
// lost), and probabilities lose up to 2^-11 of themselves, an eighth of what the output's rounding
// to bf16 costs.  fp32 queries, and their probabilities, go in as hi + lo fp16
// pairs (2^-22), two MFMAs each.  Scores are sums in fp32 (of bf16 queries of 128 |q| and less beside
// the keys' part: 2^-24 of 128 sum |q| s, whatever the keys); one above what a float holds makes its row NaN.
// Few rows: HBM-bound, a key range a workgroup, its waves a quarter each, whose (m, l, o)
// meet in LDS and, of several ranges, in a second launch.  32 requests x 8192 tokens, 32/8
// heads of 128: 83-86 us for 537 MB, 6.3 TB/s, and 5 us for the second launch; 8 x 16384 x 3
// queries in fp32 50 us, 5.4 TB/s (a third of it the two prologues' and the last
// workgroups' time).  Many rows (a prompt): a wave's products (545 cycles of the matrix cores a
// tile of 32 rows) and its exponentials and conversions (650 cycles of vector instructions) follow
// one another, and the two waves of a SIMD hide little of each other's: about 1360 cycles a tile, by
// the counters.  2048 queries on 6144 tokens 272 us, 884 TFLOP/s; each wave converting its own tiles 281,
// 64 rows a wave 525, a rescaled O every tile 1169.  Where value scales differ widely from block to
// block rows' units move more often (factors of exp(1.5 N(0, 1)): 294 us).
#include "kv8.h"
#include <math.h>
#include <type_traits>

namespace pipo {

struct Kv8Attn {
    const uint8_t *keys, *values;
    const float *scales;
    const int32_t *tables, *starts, *total;
    const void *q; void *out;
    int64_t ld_q, ld_out;
    int R, rows, W, blocks, n_kv, qpg, shift, max_len;     // block = 1 << shift
    int S, chunk;                   // key ranges of `chunk` tiles
    int groups;                     // row groups of all requests, counted from above
    int few;                        // 0, or: requests of up to so many rows are the other launch's; that one has a group a request
    float scale; int scale_e;       // of the scores, times log2(e): scale 2^scale_e
    float *part;                    // [groups][n_kv][S][16 NCT][D + 2]
};

__device__ __forceinline__ f32x4 mfma16_f16(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
// The largest of three, a NaN if there is one (which costs one instruction; fmaxf would first quiet each operand).
__device__ __forceinline__ float max3(float a, float b, float c) {
    return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c);
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
// Eight bytes u as the fp16 numbers u 2^-24, which have the bytes themselves for bits
// (the products take fp16's smallest numbers as they are).
__device__ __forceinline__ u32x4 tiny8(uint32_t a, uint32_t b) {
    return u32x4{__builtin_amdgcn_perm(0u, a, 0x0C010C00u), __builtin_amdgcn_perm(0u, a, 0x0C030C02u),
                 __builtin_amdgcn_perm(0u, b, 0x0C010C00u), __builtin_amdgcn_perm(0u, b, 0x0C030C02u)};
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

// log2 of a scale, the smallest ones too (the hardware's takes what is below 2^-126 as 0); -inf of 0.
__device__ __forceinline__ float log2_any(float x) {
    const bool tiny = x < 0x1p-64f;
    return __builtin_amdgcn_logf(tiny ? x * 0x1p64f : x) - (tiny ? 64.f : 0.f);
}

// Where a row group lies: request r's groups are numbered from start(r) * qpg / (16 NCT) + r
// on, which leaves room for the part-filled last one of every request before it.
struct RowGroup { int r, row0, n, first, last; };   // rows row0 .. of the request's n * qpg; last: its total, cut off
template <int ROWS> __device__ __forceinline__ bool find_group(const Kv8Attn &p, int f, RowGroup &g, int &total) {
    // 64 requests at a time, a lane each: the last whose groups begin at or before f
    const int lane = threadIdx.x & 63;
    int lo = 0, width = p.R;
    int64_t start = 0;
    for (;;) {
        const int step = (width + 63) >> 6, r = lo + lane * step;
        const bool in = lane * step < width;
        start = in ? min(max(p.starts[r], 0), p.rows) : 0;
        total = in && step == 1 ? p.total[r] : 0;       // (asked for together: one round trip)
        const int next = in && step == 1 ? p.starts[r + 1] : 0;
        const uint64_t upto = __ballot(in && (int)(start * p.qpg / ROWS) + r <= f);
        const int at = 63 - __builtin_clzll(upto | 1);
        lo += at * step;
        width = min(step, width - at * step);
        if (step == 1) {
            const RequestRows rr = request_rows(__builtin_amdgcn_readlane((int)start, at), __builtin_amdgcn_readlane(next, at), p.rows);
            g.first = rr.first;
            g.n = rr.n;
            total = max(__builtin_amdgcn_readlane(total, at), 0);
            break;
        }
    }
    g.r = lo;
    g.row0 = (f - (int)((int64_t)g.first * p.qpg / ROWS) - lo) * ROWS;
    g.last = min(total, p.max_len);
    return g.row0 >= 0 && g.row0 < g.n * p.qpg;
}
// The same for either launch of a call: whether this one has the group.
template <int ROWS, bool SPLIT> __device__ __forceinline__ bool own_group(const Kv8Attn &p, int f, RowGroup &g, int &total) {
    if (SPLIT && p.few) {           // group f is request f
        g.r = f;
        const RequestRows rr = request_rows(p.starts[f], p.starts[f + 1], p.rows);
        g.first = rr.first;
        g.n = rr.n;
        total = max(p.total[f], 0);
        g.row0 = 0;
        g.last = min(total, p.max_len);
        return g.n > 0 && g.n * p.qpg <= p.few;
    }
    return find_group<ROWS>(p, f, g, total) && (SPLIT || g.n * p.qpg > p.few);
}
// Tiles that the rows of a group see: up to its last token's position.
template <int ROWS> __device__ __forceinline__ int tiles_of(const Kv8Attn &p, const RowGroup &g, int total) {
    const int i = min(g.row0 + ROWS, g.n * p.qpg) - 1, seen = min(total - g.n + i / p.qpg + 1, g.last);
    return seen > 0 ? (seen + 31) >> 5 : 0;
}

// The four waves of a workgroup share a row group and cut its key range into four
// (SPLIT), or take a quarter of a group of four times the rows each, and share the tiles: each
// wave makes a quarter of a tile's bytes to operands, which all of them read from LDS.
// (Heads of 64 with two tiles of bf16 rows are held to four waves a SIMD, which costs 12 bytes of scratch where units
// move: 32 requests x 8192 tokens x 20 rows 62 us, with three waves 69.)
template <typename L, int D, int NCT, bool SPLIT>
__global__ __launch_bounds__(256, SPLIT && NCT == 2 && D == 64 && sizeof(L) == 2 ? 4 : 2) void k_kv8_attn(Kv8Attn p) {
    constexpr bool PAIR = sizeof(L) == 4, DEEP = NCT == 1;
    constexpr int ROWS = 16 * NCT, GROUP = SPLIT ? ROWS : 4 * ROWS, NC = D / 64, NT = D / 16, NV = D / 32;
    const int lane = threadIdx.x & 63, j = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    int x = blockIdx.x;
    const int head = x % p.n_kv;
    x /= p.n_kv;
    const int split = SPLIT ? x % p.S : 0;
    int f = x / p.S;
    if (!SPLIT) {
        // A prompt's later rows see more tokens and go first; where every workgroup is resident at once (two a compute
        // unit), the second half goes the other way round, so that a unit has long and short ones.
        const int n = p.groups, half = (n + 1) >> 1;
        f = n * p.n_kv <= 512 + p.n_kv && f >= half ? f - half : n - 1 - f;
    }
    RowGroup rg;
    int total;
    if (f >= p.groups || !own_group<GROUP, SPLIT>(p, f, rg, total)) return;
    const int tiles = tiles_of<GROUP>(p, rg, total);
    if (!SPLIT) rg.row0 += wave * ROWS;
    const int t_lo = split * p.chunk, t_hi = min(t_lo + p.chunk, tiles);
    if (t_lo >= t_hi && split > 0) return;
    const int n_split = tiles > 0 ? (tiles + p.chunk - 1) / p.chunk : 1;
    int ta = t_lo, tb = max(t_hi, t_lo);
    if (SPLIT) {
        const int n = tb - t_lo;
        ta = t_lo + (n * wave >> 2);
        tb = t_lo + (n * (wave + 1) >> 2);
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
        if (!PAIR) sc.y = log2_any(sc.y);
    };
    struct Tile { u32x4 k[2][NC], v[NV]; float sk, sv; bool there; };      // (sv: for bf16 queries the scale's log2)
    Tile buf[DEEP ? 2 : 1];
    int64_t off = 0;                // of the tile that load_keys was called for last
    auto load_keys = [&](Tile &to, int t) {
        const int tc = min(t, tb - 1), b = tc >> sh;
        if (b - blk0 >= 64) load_ids(b);
        const int bi = b - blk0, bid = __builtin_amdgcn_readlane(id, bi);
        off = ((((int64_t)max(bid, 0) * p.n_kv + head) << p.shift) + ((tc & ((1 << sh) - 1)) << 5)) * D;
        const u32x4 *k = (const u32x4 *)(p.keys + off) + lane;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int c = 0; c < NC; ++c) to.k[u][c] = SPLIT ? __builtin_nontemporal_load(k + (u * NC + c) * 64) : k[(u * NC + c) * 64];
        return bi;
    };
    auto load_values = [&](Tile &to) {
        const u32x4 *v = (const u32x4 *)(p.values + off) + lane;
#pragma unroll
        for (int c = 0; c < NV; ++c) to.v[c] = SPLIT ? __builtin_nontemporal_load(v + c * 64) : v[c * 64];
    };
    auto load_scales = [&](Tile &to, int bi) {
        __builtin_amdgcn_sched_barrier(0);      // (they may still be on their way when the tile is asked for)
        to.there = __builtin_amdgcn_readlane(id, bi) >= 0;
        to.sk = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(sc.x), bi));
        to.sv = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(sc.y), bi));
    };
    auto load_tile = [&](Tile &to, int t) {
        const int bi = load_keys(to, t);
        load_values(to);
        load_scales(to, bi);
    };
    // !SPLIT: this wave's pieces of the next tile, and the operands of two tiles (keys, then values)
    constexpr int OPS = 4 * NC + NT, OWN = (2 * NC + NV) / 4;
    __shared__ u32x4 s_op[SPLIT ? 1 : 2][SPLIT ? 1 : OPS][64];
    u32x4 raw[OWN];
    auto load_share = [&](int t) {
        const int tc = min(t, tb - 1), b = tc >> sh;
        if (b - blk0 >= 64) load_ids(b);
        const int bi = b - blk0, bid = __builtin_amdgcn_readlane(id, bi);
        off = ((((int64_t)max(bid, 0) * p.n_kv + head) << p.shift) + ((tc & ((1 << sh) - 1)) << 5)) * D;
#pragma unroll
        for (int u = 0; u < OWN; ++u) {
            const int piece = wave + 4 * u;
            raw[u] = *((const u32x4 *)((piece < 2 * NC ? p.keys : p.values) + off) + (piece < 2 * NC ? piece : piece - 2 * NC) * 64 + lane);
        }
        return bi;
    };
    auto put_share = [&](int at) {
#pragma unroll
        for (int u = 0; u < OWN; ++u) {
            const int piece = wave + 4 * u;
#pragma unroll
            for (int e = 0; e < 2; ++e)
                s_op[SPLIT ? 0 : at][SPLIT ? 0 : 2 * piece + e][lane] =
                    piece < 2 * NC && !PAIR ? tiny8(raw[u][2 * e], raw[u][2 * e + 1]) : widen8(raw[u][2 * e], raw[u][2 * e + 1]);
        }
    };
    if (ta < tb) load_ids(ta >> sh);
    // this lane's query rows
    u32x4 qh[NCT][NC][2], ql[NCT][NC][2];
    // A product's score is (product + cq) times the tile's scale, |p.scale| and 2^eq: powers of two are kept apart, so that
    // no part of it passes what a float holds where the score does not.
    int eq[NCT];
    float cq[NCT], far_sk = INFINITY;       // (the key scale above which a score may pass 2^22)
    int seen[NCT];                  // tokens it sees
    const float sign = p.scale < 0.f ? -1.f : 1.f;
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct) {
        const int rr = rg.row0 + 16 * ct + j, i = rr / p.qpg, h = head * p.qpg + rr - i * p.qpg;
        const bool is = i < rg.n;
        seen[ct] = is ? max(min(total - rg.n + i + 1, rg.last), 0) : 0x7FFFFFFF;    // (what is no row is not written)
        float v[NC][16];
        const L *q = (const L *)p.q + (is ? (rg.first + i) * p.ld_q + (int64_t)h * D + 16 * g : 0);
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
        // the power of two that brings the largest to [2^14, 2^15) (of none: one with which no score is far)
        const int ex = top > 0.f && top < INFINITY ? 14 - ilogbf(top) : 100;
        eq[ct] = p.scale_e - ex;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
#pragma unroll
            for (int e = 0; e < 16; ++e) v[c][e] = ldexpf(v[c][e], ex) * sign;
            fp16_8<PAIR>(v[c], qh[ct][c][0], ql[ct][c][0]);
            fp16_8<PAIR>(v[c] + 8, qh[ct][c][1], ql[ct][c][1]);
        }
        cq[ct] = 0.f;
        if (!PAIR) {                // the keys go in as u 2^-24, not u - 128
            float sum = 0.f;
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int k = 0; k < 4; ++k) sum += f16_lo(qh[ct][c][e][k]) + f16_hi(qh[ct][c][e][k]);
            cq[ct] = -0x1p-17f * col_sum(sum);
            eq[ct] += 24;
        }
        // (products and cq reach 2^22 D, and with keys as u 2^-24 D)
        far_sk = fminf(far_sk, ldexpf((PAIR ? 1.f : 0x1p22f) / (D * fabsf(p.scale)), -eq[ct]));
        __builtin_amdgcn_sched_barrier(0);      // (one after the other, or their floats do not fit)
    }
    far_sk = __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(-wave_max_dpp(-far_sk))));
    int all_see = 0x7FFFFFFF;       // tokens that every row sees
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct) all_see = min(all_see, seen[ct]);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) all_see = min(all_see, __shfl_xor(all_see, o));
    all_see = __builtin_amdgcn_readfirstlane(all_see);

    // A row's O is in units of 2^unit; probabilities as 2^8 exp2(s - m), where m, a row's reference, follows its
    // maximum only when that is more than 4 above it: O is seldom rescaled, and 2^15 at most goes into fp16.  Pairs
    // take 2^14 and the maximum itself: the lower half of a small probability has fp16's smallest step (errors of the
    // whole, 8 x 16384 tokens: 3.9e-6 with 2^8, 5e-7).  So what is small beside the row's largest loses up to 2^-33 of
    // that (pairs: 2^-39).
    constexpr float kUp = PAIR ? 14.f : 8.f, kSlack = PAIR ? 0.f : 4.f, kMost = PAIR ? 1.f : 3.f;
    f32x4 o[NCT][NT];
    float m_run[NCT], l_run[NCT], unit[NCT];
    float unit0 = __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(sc.y)));     // the first block's value scale, or any
    unit0 = floorf(PAIR ? log2_any(unit0) : unit0) + 1.f;
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct) {
        m_run[ct] = -INFINITY;
        l_run[ct] = 0.f;
        unit[ct] = fabsf(unit0) < 200.f ? unit0 : 0.f;
#pragma unroll
        for (int t = 0; t < NT; ++t) o[ct][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    typedef f32x4 Scores[NCT][2];
    auto score = [&](const Tile &b, Scores &st, int share) {
        u32x4 ka[SPLIT ? 1 : 4 * NC];
        if constexpr (!SPLIT) {
#pragma unroll
            for (int i = 0; i < 4 * NC; ++i) ka[i] = s_op[share][i][lane];
            __builtin_amdgcn_sched_barrier(0);
        }
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
                    const u32x4 a = !SPLIT ? ka[SPLIT ? 0 : (u * NC + c) * 2 + e]
                                    : PAIR ? widen8(b.k[u][c][2 * e], b.k[u][c][2 * e + 1])
                                           : tiny8(b.k[u][c][2 * e], b.k[u][c][2 * e + 1]);
#pragma unroll
                    for (int ct = 0; ct < NCT; ++ct) {
                        st[ct][u] = mfma16_f16(a, qh[ct][c][e], st[ct][u]);
                        if (PAIR) st[ct][u] = mfma16_f16(a, ql[ct][c][e], st[ct][u]);
                    }
                }
    };
    // A tile whose value scale is far from the rows' units: where it is to be seen in O beside what is there, the row's unit
    // moves so that both can be held.  r: its largest score less the row's reference, in all of a row's lanes alike.
    //   Up, where its probabilities times its scale would not go into fp16 (fp32: weigh more than 2^4), or what is there
    // stays large enough (2^8) beside their smallest steps.  Down, as far as what is there keeps below 2^81 (more than
    // that, and the tile is nothing beside it); what has lost its weight by its scores does not hold a unit up.
    // fold: what the probabilities' exponents get; apart: they are too small then to be summed for l as well.
    auto settle = [&](const Tile &b, const float (&mx)[NCT], float (&fold)[NCT], float (&kv)[NCT]) __attribute__((always_inline)) {
        bool apart = false;
        const float ls = PAIR ? log2_any(b.sv) : b.sv;
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct) {
            const float r = col_max(mx[ct]) - m_run[ct], d = ls - unit[ct], least = PAIR ? r + d : d;
            float top = 0.f;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int v = 0; v < 4; ++v) top = fmaxf(top, fabsf(o[ct][t][v]));
            top = col_max(top);
            const float held = top > 0.f ? (float)ilogbf(top) : -1000.f;
            float to = unit[ct];
            if (r > -INFINITY) {        // (a row that sees nothing of it stays as it is, and so with a NaN)
                if (r + d > (PAIR ? 4.f : 7.f)) to = fmaxf(to, ceilf(ls + fminf(r, 0.f) - kMost));
                else if (d > kMost && held - d >= 8.f) to = ceilf(ls - kMost);
                else if (least < (PAIR ? -60.f : -3.f) && ls > -INFINITY)
                    to = fminf(to, fmaxf(floorf(PAIR ? ls + r : ls + 3.f), to + held - 80.f));
            }
            const int up = (int)(unit[ct] - to);
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int v = 0; v < 4; ++v) o[ct][t][v] = ldexpf(o[ct][t][v], up);
            unit[ct] = to;
            fold[ct] = ls - to;
            apart |= fold[ct] < -3.f && r > -INFINITY;
            if (PAIR) {                 // (a tile of small weight and a large scale needs its probabilities' lower bits)
                fold[ct] = r > -INFINITY ? fminf(ceilf(-r), 1000.f) : 0.f;
                kv[ct] = ldexpf(b.sv, (int)(-to - fold[ct]));
            }
        }
        return !PAIR && __builtin_amdgcn_ballot_w64(apart) != 0;
    };
    // A tile's probabilities, and what they add to l and O.
    auto tile_as = [&](const Tile &b, int t0, const Scores &st, int share, auto all) __attribute__((always_inline)) {
        constexpr bool whole = decltype(all)::value;    // every row sees all of it
        if (!b.there) return;       // no such block: its tokens are not there
        u32x4 va[SPLIT ? 1 : NT];
        if constexpr (!SPLIT) {     // asked for before the exponentials
#pragma unroll
            for (int d = 0; d < NT; ++d) va[d] = s_op[share][4 * NC + d][lane];
            __builtin_amdgcn_sched_barrier(0);
        }
        float s[NCT][8], mx[NCT], fk[NCT], ck[NCT];
        bool rise = false;
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct) {
            fk[ct] = ldexpf(b.sk, eq[ct]) * fabsf(p.scale);
            ck[ct] = cq[ct] * fk[ct];
#pragma unroll
            for (int k = 0; k < 8; ++k) s[ct][k] = st[ct][k >> 2][k & 3];
        }
        auto hidden = [&](int ct, int k) { return t0 + 16 * (k >> 2) + 4 * g + (k & 3) >= seen[ct]; };
        auto max8 = [](const float *v) { return max3(max3(v[0], v[1], v[2]), max3(v[3], v[4], v[5]), max3(v[6], v[7], v[7])); };
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct) {
            if (whole) {
                mx[ct] = fmaf(max8(s[ct]), fk[ct], ck[ct]);
            } else {
                float v[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = hidden(ct, k) ? -INFINITY : s[ct][k];
                mx[ct] = max8(v);
                mx[ct] = mx[ct] == -INFINITY ? mx[ct] : fmaf(mx[ct], fk[ct], ck[ct]);   // (a scale of 0 times it is no number)
            }
            rise |= mx[ct] > m_run[ct] + kSlack;
        }
        if (__builtin_amdgcn_ballot_w64(rise)) {
#pragma unroll
            for (int ct = 0; ct < NCT; ++ct) {
                const float m = fmaxf(m_run[ct], col_max(mx[ct]));
                const float al = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run[ct] - m);
                m_run[ct] = m;
                l_run[ct] *= al;
#pragma unroll
                for (int d = 0; d < NT; ++d) o[ct][d] *= al;
            }
        }
        // The tile's scale, over the row's unit, goes into its probabilities.  (Pairs: into what the tile adds, by an fma,
        // which rounds to nearest.)
        float fold[NCT], kv[NCT];
        bool odd = false, apart = false;
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct) ck[ct] -= m_run[ct] == -INFINITY ? -kUp : m_run[ct] - kUp;
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct) {
            if (PAIR) {
                fold[ct] = 0.f;
                kv[ct] = ldexpf(b.sv, -(int)unit[ct]);
                odd |= kv[ct] < 0x1p-60f || kv[ct] > 0x1p8f;
            } else {
                fold[ct] = b.sv - unit[ct];
                odd |= fabsf(fold[ct]) > 3.f;
            }
        }
        // (said to be rare, so that its registers are not kept from the others': 2048 queries on 6144 tokens 272 us, else 280)
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(odd || b.sk > far_sk) != 0, 0)) {
            apart = settle(b, mx, fold, kv);
            // A score's exponent is one fma from the products on, s fk + (ck - m): exact where it counts, as long as the
            // roundings of ck and m are small.  Where scores may pass 2^22 they are rounded by themselves, as m was, so
            // that the largest is m and no exponent comes out far above it.
            if (b.sk > far_sk) {
#pragma unroll
                for (int ct = 0; ct < NCT; ++ct) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) s[ct][k] = fmaf(s[ct][k], fk[ct], cq[ct] * fk[ct]) - (m_run[ct] == -INFINITY ? 0.f : m_run[ct]);
                    fk[ct] = 1.f;
                    ck[ct] = kUp;
                }
            }
        }
        u32x4 ph[NCT], pl[NCT];
        f32x4 w[NCT];
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct) {
            const float c = ck[ct] + fold[ct];
            const u32x4 ones{0x3C003C00u, 0x3C003C00u, 0x3C003C00u, 0x3C003C00u};
            if (__builtin_expect(apart, 0)) {       // l from probabilities without the scale
                float e[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    e[k] = __builtin_amdgcn_exp2f(fmaf(s[ct][k], fk[ct], ck[ct]));
                    if (!whole && hidden(ct, k)) e[k] = 0.f;
                }
                fp16_8<false>(e, ph[ct], pl[ct]);
                w[ct] = mfma16_f16(ones, ph[ct], f32x4{0.f, 0.f, 0.f, 0.f});
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) s[ct][k] = __builtin_amdgcn_exp2f(fmaf(s[ct][k], fk[ct], c));
            if (!whole) {
#pragma unroll
                for (int k = 0; k < 8; ++k) s[ct][k] = hidden(ct, k) ? 0.f : s[ct][k];
            }
            fp16_8<PAIR>(s[ct], ph[ct], pl[ct]);
            // their sum, over the tile's tokens: from the matrix cores, where they have been rounded
            if (!apart) w[ct] = mfma16_f16(ones, ph[ct], f32x4{0.f, 0.f, 0.f, 0.f});
            if (PAIR) w[ct] = mfma16_f16(ones, pl[ct], w[ct]);
        }
#pragma unroll
        for (int d = 0; d < NT; ++d) {
            const u32x4 a = !SPLIT ? va[SPLIT ? 0 : d] : widen8(b.v[d >> 1][2 * (d & 1)], b.v[d >> 1][2 * (d & 1) + 1]);
#pragma unroll
            for (int ct = 0; ct < NCT; ++ct) {
                if constexpr (PAIR) {
                    f32x4 x = mfma16_f16(a, ph[ct], f32x4{0.f, 0.f, 0.f, 0.f});
                    x = mfma16_f16(a, pl[ct], x);
                    const float k = t0 < seen[ct] ? kv[ct] : 0.f;    // (a row that sees nothing of the tile gets no NaN from it)
#pragma unroll
                    for (int v = 0; v < 4; ++v) o[ct][d][v] = fmaf(x[v], k, o[ct][d][v]);
                } else {
                    o[ct][d] = mfma16_f16(a, ph[ct], o[ct][d]);
                }
            }
        }
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct)    // (finite whatever the scale: a row that sees nothing of the tile adds 0 times it)
            l_run[ct] = fmaf(w[ct][0], apart ? 1.f : __builtin_amdgcn_exp2f(fminf(-fold[ct], 100.f)), l_run[ct]);
    };
    if (ta < tb) {
        Scores st;
        int t = ta;
        const int tw = all_see >> 5;            // tiles before this one are seen whole
        if constexpr (!SPLIT) {
            Tile &now = buf[0], next{};
            int bi = load_share(t);
            load_scales(now, bi);
            put_share(0);
            bi = load_share(t + 1);
            load_scales(next, bi);
            __syncthreads();
            int at = 0;
            auto one = [&](auto all) {
                score(now, st, at);
                put_share(at ^ 1);              // (nobody reads it since the last barrier)
                bi = load_share(t + 2);
                tile_as(now, t * 32, st, at, all);
                now.there = next.there;
                now.sk = next.sk;
                now.sv = next.sv;
                load_scales(next, bi);
                __syncthreads();
                at ^= 1;
                ++t;
            };
            while (t < min(tb, tw)) one(std::true_type{});
            while (t < tb) one(std::false_type{});
        } else if constexpr (DEEP) {            // two tiles on their way
            load_tile(buf[0], ta);
            load_tile(buf[1], ta + 1);
            auto two = [&](auto all) {
                score(buf[0], st, 0);
                tile_as(buf[0], t * 32, st, 0, all);
                load_tile(buf[0], t + 2);
                score(buf[1], st, 0);
                tile_as(buf[1], t * 32 + 32, st, 0, all);
                load_tile(buf[1], t + 3);
                t += 2;
            };
            while (t + 2 < min(tb, tw + 1)) two(std::true_type{});
            while (t + 2 < tb) two(std::false_type{});
            score(buf[0], st, 0);
            tile_as(buf[0], t * 32, st, 0, std::false_type{});
            if (t + 1 < tb) {
                score(buf[1], st, 0);
                tile_as(buf[1], t * 32 + 32, st, 0, std::false_type{});
            }
        } else {                    // the next tile's keys while this one's values are used, its values while its keys are
            load_tile(buf[0], ta);
            auto one = [&](auto all) {
                score(buf[0], st, 0);
                const int bi = load_keys(buf[0], t + 1);
                tile_as(buf[0], t * 32, st, 0, all);
                load_values(buf[0]);
                load_scales(buf[0], bi);
                ++t;
            };
            while (t < min(tb, tw)) one(std::true_type{});
            while (t < tb) one(std::false_type{});
        }
    }
    // O over l, so that no sum of values passes the largest of them
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct) {
        const float inv = l_run[ct] == 0.f ? 0.f : 1.f / l_run[ct];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int v = 0; v < 4; ++v) o[ct][t][v] = ldexpf(o[ct][t][v] * inv, (int)unit[ct]);
    }
    // row rr of the group: to the output, or as a record (average, m, l) for the others of its key ranges
    auto finish = [&](int rr, int d, float a, float b, float c, float e, float m, float l) {
        const int at = rg.row0 + rr, i = at / p.qpg;
        if (i >= rg.n) return;
        if (n_split == 1) {
            L *to = (L *)p.out + (rg.first + i) * p.ld_out + (int64_t)(head * p.qpg + at - i * p.qpg) * D + d;
            Piece<L>::put(to, a);
            Piece<L>::put(to + 1, b);
            Piece<L>::put(to + 2, c);
            Piece<L>::put(to + 3, e);
        } else {
            float *rec = p.part + ((((int64_t)f * p.n_kv + head) * p.S + split) * ROWS + rr) * (D + 2);
            *(float2 *)(rec + d) = make_float2(a, b);
            *(float2 *)(rec + d + 2) = make_float2(c, e);
            if (d == 0) *(float2 *)(rec + D) = make_float2(m, l);
        }
    };
    if constexpr (!SPLIT) {
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
            for (int t = 0; t < NT; ++t)
                finish(16 * ct + j, 16 * t + 4 * g, o[ct][t][0], o[ct][t][1], o[ct][t][2], o[ct][t][3], m_run[ct], l_run[ct]);
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
                const int rr = e / (D / 4), d = e % (D / 4) * 4;
                float M = -INFINITY, l = 0.f, k[4], a[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < 4; ++w) M = fmaxf(M, red[w][rr][D]);
                const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    k[w] = __builtin_amdgcn_exp2f(red[w][rr][D] - ref) * red[w][rr][D + 1];
                    l += k[w];
                }
                const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
                for (int w = 0; w < 4; ++w)
#pragma unroll
                    for (int v = 0; v < 4; ++v) a[v] += k[w] * inv * red[w][rr][d + v];
                finish(16 * ct + rr, d, a[0], a[1], a[2], a[3], M, l);
            }
        }
    }
}

// The key ranges' records of a row as one: a wave a row, D / 64 dimensions a lane, a lane a range's weight.  Where
// a row's records lie does not hang on whose row it is: the first ones are asked for along with the lengths.
template <typename L, int D, int NCT> __global__ __launch_bounds__(256) void k_kv8_attn_join(Kv8Attn p) {
    constexpr int ROWS = 16 * NCT, E = D / 64, U = 16;
    typedef __attribute__((ext_vector_type(E))) float vec;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int head = blockIdx.x % p.n_kv, f = blockIdx.x / p.n_kv;
    const float *records = p.part + ((int64_t)f * p.n_kv + head) * p.S * ROWS * (D + 2);
    const int64_t step = (int64_t)ROWS * (D + 2);
    auto stat = [&](int rr, int s) { return s < p.S ? *(const float2 *)(records + s * step + rr * (D + 2) + D) : make_float2(0.f, 0.f); };
    auto ask = [&](vec (&v)[U], int rr, int s) {
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = *(const vec *)(records + min(s + u, p.S - 1) * step + rr * (D + 2) + lane * E);
    };
    vec v[U];
    float2 ml = stat(wave, lane);
    ask(v, wave, 0);
    RowGroup rg;
    int total;
    if (!own_group<ROWS, true>(p, f, rg, total)) return;
    const int tiles = tiles_of<ROWS>(p, rg, total);
    const int n = (tiles + p.chunk - 1) / p.chunk;
    if (n <= 1) return;             // the unit wrote it out itself
    for (int rr = wave; rr < ROWS && rg.row0 + rr < rg.n * p.qpg; rr += 4) {
        if (rr != wave) {
            ml = stat(rr, lane);
            ask(v, rr, 0);
        }
        float M = -INFINITY, l = 0.f;
        vec a = 0.f;
        for (int s0 = 0; s0 < n; s0 += 64) {
            if (s0 > 0) ml = stat(rr, s0 + lane);
            const float mine = s0 + lane < n ? ml.x : -INFINITY;
            const float m = fmaxf(M, wave_max_dpp(mine)), ref = m == -INFINITY ? 0.f : m;
            float k = s0 + lane < n ? __builtin_amdgcn_exp2f(mine - ref) * ml.y : 0.f;
            const float before = l * __builtin_amdgcn_exp2f(M - ref);
            l = before + wave_sum_dpp(k);
            const float inv = l == 0.f ? 0.f : 1.f / l;
            a *= before * inv;          // (averages, weighed by their part of l)
            k *= inv;
            M = m;
            const int cnt = min(n - s0, 64);
            for (int s = 0; s < cnt; s += U) {
                if (s0 + s > 0) ask(v, rr, s0 + s);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const float w = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(k), min(s + u, 63)));
                    if (s + u < cnt) a += w * v[u];
                }
            }
        }
        const int i = (rg.row0 + rr) / p.qpg, h = head * p.qpg + rg.row0 + rr - i * p.qpg;
        L *to = (L *)p.out + (rg.first + i) * p.ld_out + (int64_t)h * D + lane * E;
#pragma unroll
        for (int e = 0; e < E; ++e) Piece<L>::put(to + e, a[e]);
    }
}

// ---- shapes of a launch ----------------------------------------------------------------
// Tiles of rows a wave (nct), key ranges or shared tiles (split), row groups; S ranges of `chunk` tiles: of the launch
// or, beside one of shared tiles, of the second one for requests of few rows.
constexpr int kFewRows = 32;
struct Kv8Shape { int nct, groups, S, chunk; bool split, second; int64_t part; };

// Key ranges that fill the chip in whole rounds.  A unit takes its prologue (about as long as three tiles of a wave) and
// a quarter of its tiles, a joining launch eight and what it reads.  slots: workgroups that the compute units hold by their
// registers.  (32 x 8192 tokens, 256 units, 768 slots, in 3 / 4 / 8 / 12 ranges: 89 / 95 / 95 / 100 us.)
static int key_ranges(int64_t units, int tiles, int slots) {
    int best_S = 1;
    double best = 1e300;
    for (int S = 1; S <= 64 && 4 * S <= tiles + 3; ++S) {
        const int64_t rounds = (units * S + slots - 1) / slots;
        const double t = (double)rounds * (((tiles + S - 1) / S + 3) / 4 + 3) + (S > 1 ? 8. + S / 16. : 0.);
        if (t < best) { best = t; best_S = S; }
    }
    return best_S;
}
static Kv8Shape shape_of(int R, int rows, int n_q, int n_kv, int D, int max_len, bool work) {
    Kv8Shape s{};
    const int qpg = n_q / n_kv, tiles = (max_len + 31) / 32;
    const int64_t per = ((int64_t)(rows + R - 1) / R) * qpg;        // query rows of a request and KV head, on average
    s.nct = per <= 16 ? 1 : 2;
    const int64_t tile_rows = 16 * s.nct;
    int64_t units = (int64_t)R * ((per + tile_rows - 1) / tile_rows) * n_kv;
    // Tiles are shared by waves of different rows where there are rows for two waves at least and units for every SIMD.
    // A batch may still hold requests of a few rows and many tokens (decoding ones beside prompts), whose tokens one
    // workgroup would take one after the other: they get key ranges, in a launch of their own.  Few are as many rows as
    // a unit of that launch holds (a number that comes from the kernel; requests of more rows have not been timed there).
    s.split = per < 64 || units < 1024;
    s.second = !s.split && R > 1;
    s.groups = (int)((int64_t)rows * qpg / (s.split ? tile_rows : 4 * tile_rows)) + R;
    if (s.second) units = (int64_t)R * n_kv;
    s.S = work && (s.split || s.second) ? key_ranges(units, tiles, 256 * (D == 64 ? (s.nct == 1 ? 4 : 3) : (s.nct == 1 ? 3 : 2))) : 1;
    s.chunk = (tiles + s.S - 1) / s.S;
    s.S = (tiles + s.chunk - 1) / s.chunk;
    s.part = s.S > 1 ? (int64_t)(s.second ? R : s.groups) * n_kv * s.S * tile_rows * (D + 2) * 4 : 0;
    return s;
}

template <typename L, int D, int NCT> static bool run_split(const Kv8Attn &p, hipStream_t s) {
    return launch(k_kv8_attn<L, D, NCT, true>, (unsigned)((int64_t)p.groups * p.S * p.n_kv), 256, 0, s, p) &&
           (p.S == 1 || launch(k_kv8_attn_join<L, D, NCT>, (unsigned)(p.groups * p.n_kv), 256, 0, s, p));
}
template <typename L, int D> static bool run_attn(const Kv8Attn &p, const Kv8Shape &s, hipStream_t st) {
    if (s.split) return s.nct == 1 ? run_split<L, D, 1>(p, st) : run_split<L, D, 2>(p, st);
    Kv8Attn rows = p;               // (all of a row's tokens: one range)
    rows.S = 1;
    rows.chunk = (p.max_len + 31) / 32;
    rows.few = s.second ? kFewRows : 0;
    if (!launch(k_kv8_attn<L, D, 2, false>, (unsigned)(p.groups * p.n_kv), 256, 0, st, rows)) return false;
    Kv8Attn ranges = p;
    ranges.groups = p.R;
    ranges.few = kFewRows;
    return !s.second || run_split<L, D, 2>(ranges, st);
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
    // The output may take the queries' place: a row's heads are read by the workgroup that writes them, before it does, or
    // by those that leave them to the joining launch.
    if (!same_or_apart(q, ld_q, out, ld_out, rows, least, sizeof(L))) return PIPO_EINVAL;
    const Kv8Shape s = shape_of(R, rows, n_q, c->n_kv, c->head_dim, max_len, work != nullptr);
    if (work && s.part > 0 && (!kv8_aligned(work, 16) || work_bytes < s.part)) return PIPO_EINVAL;
    int scale_e;
    const float scale_m = (float)frexp(scale * 1.4426950408889634074, &scale_e);
    Kv8Attn p{c->keys, c->values, c->scales, tables, starts, total, q, out, ld_q, ld_out, R, rows, width, c->blocks,
              c->n_kv, n_q / c->n_kv, __builtin_ctz((unsigned)c->block), max_len, s.S, s.chunk, s.groups, 0,
              scale_m, scale_e, (float *)work};
    hipStream_t st = (hipStream_t)stream;
    return (c->head_dim == 128 ? run_attn<L, 128>(p, s, st) : run_attn<L, 64>(p, s, st)) ? PIPO_OK : PIPO_EHIP;
}

}  // namespace pipo

using namespace pipo;

extern "C" int64_t pipo_kv8_attention_work_bytes(const pipo_kv8 *c, int32_t R, int32_t rows, int32_t n_q, int32_t max_len,
                                                 int32_t bf16) {
    if (!attn_sizes_ok(c, R, rows, n_q, max_len) || rows == 0) return 0;
    return shape_of(R, rows, n_q, c->n_kv, c->head_dim, max_len, true).part;
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
