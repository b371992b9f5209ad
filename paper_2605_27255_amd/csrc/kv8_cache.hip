// The paged 8-bit cache: blocks and slots of a step's tokens, keys and values into
// the cache, and back.
#include "kv8.h"

namespace pipo {

bool kv8_ok(const pipo_kv8 *c) {
    return c && kv8_aligned(c->keys, 16) && kv8_aligned(c->values, 16) && kv8_aligned(c->scales, 8) && c->blocks >= 1 &&
           c->n_kv >= 1 && c->n_kv <= 256 && (c->head_dim == 64 || c->head_dim == 128) &&
           (c->block == 32 || c->block == 64 || c->block == 128 || c->block == 256) &&
           (int64_t)c->blocks * c->block < (int64_t)1 << 31;
}

// ---- blocks and slots --------------------------------------------------------------
struct PlanParams {
    int R, W, block, blocks;
    const int32_t *lens, *add;
    int32_t *tables, *held, *stack, *n_free;
    int rows;
    int32_t *starts, *total, *slots, *positions;
    int fill;                       // the rows are written by the planning workgroup itself
};

// Exclusive sums of a and b over the workgroup's threads; A and B get the totals.
template <int NT> __device__ __forceinline__ void scan2(int &a, int &b, int &A, int &B, int (*s_w)[NT / 64]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int x = a, y = b;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(x, o), v = __shfl_up(y, o);
        if (lane >= o) { x += u; y += v; }
    }
    __syncthreads();
    if (lane == 63) { s_w[0][wave] = x; s_w[1][wave] = y; }
    __syncthreads();
    int p = 0, q = 0;
    A = B = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
        const int u = s_w[0][w], v = s_w[1][w];
        if (w < wave) { p += u; q += v; }
        A += u;
        B += v;
    }
    a = p + x - a;
    b = q + y - b;
}

__device__ __forceinline__ void put_row(const PlanParams &p, int row, int r, int from, int to, int total, int last) {
    int slot = -1, pos = -1;
    if (row < last && total > 0) {
        pos = total - (to - row);
        const int at = p.tables[(int64_t)r * p.W + pos / p.block];
        if ((unsigned)at < (unsigned)p.blocks) slot = at * p.block + pos % p.block; else pos = -1;
    }
    p.slots[row] = slot;
    p.positions[row] = pos;
}

// One workgroup, a request a thread (NT at a time), then a block a thread: sums over
// the requests give each its place in the stack and its rows.  Latency-bound: three
// dependent rounds of loads (lengths, stack, table) and the sums' barriers (32
// requests of two tokens 4 us, 256 prompts of 2144 blocks 8.4 and their 129000 rows 3.4).
template <int NT> __global__ __launch_bounds__(NT) void k_kv8_plan(PlanParams p) {
    __shared__ int s_w[2][NT / 64], s_pref[NT + 1], s_held[NT], s_start[NT + 1], s_total[NT], s_take;
    const int tid = threadIdx.x;
    auto held_of = [&](int r) { return r < p.R ? min(max(p.held[r], 0), p.W) : 0; };
    auto find = [&](int n, int e) {     // the last of n requests whose sum before it is at most e
        int lo = 0, hi = n;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (s_pref[mid] <= e) lo = mid; else hi = mid;
        }
        return lo;
    };
    int64_t avail = min(max(p.n_free[0], 0), p.blocks);
    // what the requests that ended give back
    int64_t back_all = 0;
    for (int c0 = 0; c0 < p.R; c0 += NT) {
        const int r = c0 + tid;
        int back = r < p.R && p.add[r] < 0 ? held_of(r) : 0, none = 0, all, z;
        scan2<NT>(back, none, all, z, s_w);
        back_all += all;
    }
    if (back_all > 0) {
        int64_t before = 0;
        for (int c0 = 0; c0 < p.R; c0 += NT) {
            const int r = c0 + tid;
            int back = r < p.R && p.add[r] < 0 ? held_of(r) : 0, none = 0, all, z;
            scan2<NT>(back, none, all, z, s_w);
            s_pref[tid] = back;
            __syncthreads();
            for (int e = tid; e < all; e += NT) {
                const int i = find(NT, e);
                int32_t *entry = p.tables + (int64_t)(c0 + i) * p.W + (e - s_pref[i]);
                const int64_t to = avail + back_all - 1 - (before + e);
                if (to < p.blocks) p.stack[to] = *entry;    // (more than there are: the caller's counts are wrong)
                *entry = -1;
            }
            before += all;
            __syncthreads();
        }
        avail = avail + back_all < p.blocks ? avail + back_all : p.blocks;
    }
    // blocks for the others
    int64_t taken = 0, wanted = 0;
    int rows_before = 0;
    for (int c0 = 0; c0 < p.R; c0 += NT) {
        const int r = c0 + tid;
        const int add = r < p.R ? p.add[r] : -1, len = r < p.R ? p.lens[r] : 0, h = add < 0 ? 0 : held_of(r);
        const int n = min(max(add, 0), kKv8MaxRows + 1);
        const int64_t want = ((int64_t)len + max(add, 0) + p.block - 1) / p.block;
        const bool valid = add >= 0 && len >= 0 && want <= p.W;
        const int need = valid ? max((int)want - h, 0) : 0;
        int nb = need, nr = n, all_b, all_r;
        scan2<NT>(nb, nr, all_b, all_r, s_w);
        const int64_t from = (int64_t)rows_before + nr;     // (a sum of at most NT (2^20 + 1) and 2^20 + 1)
        const bool fits = valid && (need == 0 || wanted + nb + need <= avail) && from + n <= p.rows;
        if (tid == 0) s_take = 0;
        s_pref[tid] = nb;
        s_held[tid] = h;
        __syncthreads();
        if (fits && need > 0) atomicMax(&s_take, nb + need);    // (behind the first that finds none, none takes any)
        const int start = (int)(from < p.rows ? from : p.rows), total = fits ? len + add : 0;
        if (r < p.R) {
            p.starts[r] = start;
            p.total[r] = total;
            if (add < 0 || fits) p.held[r] = h + (fits ? need : 0);
        }
        s_start[tid] = start;
        s_total[tid] = total;
        __syncthreads();
        const int take = s_take;
        for (int e = tid; e < take; e += NT) {
            const int i = find(NT, e);
            p.tables[(int64_t)(c0 + i) * p.W + s_held[i] + (e - s_pref[i])] = p.stack[avail - 1 - (wanted + e)];
        }
        taken += take;
        wanted += all_b;
        rows_before = (int)min((int64_t)rows_before + all_r, (int64_t)kKv8MaxRows + 1);
    }
    const int last = min(rows_before, p.rows);
    if (tid == 0) {
        p.starts[p.R] = last;
        p.n_free[0] = (int)(avail - taken);
        s_start[min(p.R, NT)] = last;
    }
    if (!p.fill) return;
    __syncthreads();
    for (int row = tid; row < p.rows; row += NT) {      // (R <= NT)
        const int r = request_of(s_start, p.R, row);
        put_row(p, row, r, s_start[r], s_start[r + 1], s_total[r], last);
    }
}
// The rows of a step of many tokens.
__global__ __launch_bounds__(256) void k_kv8_rows(PlanParams p) {
    constexpr int kInLds = 4096;
    __shared__ int s_start[kInLds + 1];
    const int row = blockIdx.x * 256 + threadIdx.x;
    const int32_t *starts = p.starts;
    if (p.R <= kInLds) {
        for (int i = threadIdx.x; i <= p.R; i += 256) s_start[i] = p.starts[i];
        __syncthreads();
        starts = s_start;
    }
    if (row >= p.rows) return;
    const int r = request_of(starts, p.R, row);
    put_row(p, row, r, starts[r], starts[r + 1], p.total[r], starts[p.R]);
}

// ---- keys and values into the cache ---------------------------------------------------
template <typename L> struct AppendParams {
    const L *x[2]; int64_t ld[2];   // keys, values
    uint8_t *store[2];
    float *scales;
    const int32_t *slots;
    int rows, chunk, blocks, n_kv, D, shift;    // block = 1 << shift
};

// Sixteen x / s rounded to nearest even, as bytes 128 + x / s: the product with 1 / s
// rounded, unless what that leaves, which one fma gives exactly, is half a step or more.
__device__ __forceinline__ u32x4 round16(const float *x, float s, float inv) {
    float q[16];
    const float h = 0.5f * s;
    bool near = false;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        q[i] = rintf(x[i] * inv);
        near |= fabsf(fmaf(-q[i], s, x[i])) >= h;
    }
    if (near) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float e = fmaf(-q[i], s, x[i]), a = fabsf(e);
            if (a > h || (a == h && ((int)q[i] & 1))) q[i] += copysignf(1.f, e);
        }
    }
    u32x4 w{0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 16; ++i) w[i >> 2] = __builtin_amdgcn_cvt_pk_u8_f32(q[i] + 128.f, i & 3, w[i >> 2]);
    return w;
}
// q old / s likewise, in 64 bits: the product has more digits than a float.
__device__ __forceinline__ int round_again(int u, double old, double s, double inv) {
    const double x = (double)(u - 128) * old;
    double q = rint(x * inv);
    const double e = fma(-q, s, x), a = fabs(e), h = 0.5 * s;
    if (a > h || (a == h && ((int)q & 1))) q += copysign(1., e);
    return 128 + (int)q;
}

// A workgroup takes the blocks whose first row is among `chunk` rows, of one head, keys
// or values: their largest magnitude, the scale, and the tiles with new bytes.  An item
// is 16 dimensions of a token.  Rows that follow one another as their slots do, as a
// rule, are found by their number; others by a table of tokens (of rows with one slot the
// last), and so are runs with rows among them that have no slot.  Bound by latency at a step's single tokens (32 in 6.8 us: slots, rows and scale,
// the old tile, one after the other), at a prompt's by how many workgroups a compute unit
// holds (8192 tokens of 8 heads x 128: 22 us, 2.3 TB/s in and out).
template <typename L, int NT> __global__ __launch_bounds__(NT, 4) void k_kv8_append(AppendParams<L> p) {
    constexpr int N = Piece<L>::N, KEEP = 2;    // items of a thread that stay in registers
    extern __shared__ __align__(16) uint8_t s_stage[];      // values: [token][D + 16] bytes, in pieces of 16
    __shared__ int s_row[256], s_near[2];
    __shared__ uint32_t s_top[NT / 64];
    const int tid = threadIdx.x, lane = tid & 63, head = blockIdx.y, which = blockIdx.z;
    const int B = 1 << p.shift, D = p.D, E = D >> 4, pitch = D + 16;
    const L *x = p.x[which] + (int64_t)head * D;
    const int64_t ld = p.ld[which];
    const int from = blockIdx.x * p.chunk, upto = min(from + p.chunk, p.rows);
    auto slot_of = [&](int i) { return i >= 0 && i < p.rows ? p.slots[i] : -1; };
    auto block_of = [&](int slot) { return slot >= 0 && (slot >> p.shift) < p.blocks ? slot >> p.shift : -1; };
    // The nearest row from `at` on (up: 1, down: -1) that has a slot, and its block (-1: there is none), by the whole
    // workgroup, all of whose waves see the same slots and call this together: a step's padding may be long (32 tokens
    // and 65504 rows without a slot: 114 us a call, of them 94 for the launch; where each wave searches alone, 188).
    auto seek = [&](int at, int up, int &row) {
        constexpr int U = 16, NONE = 0x7FFFFFFF;
        __syncthreads();
        if (tid < 2) s_near[tid] = NONE;
        __syncthreads();
#pragma unroll 1
        for (int step = 0; at >= 0 && at < p.rows; ++step, at += up * U * NT) {
            int s[U], near = NONE;
#pragma unroll
            for (int u = 0; u < U; ++u) s[u] = slot_of(at + up * (u * NT + tid));
#pragma unroll
            for (int u = U - 1; u >= 0; --u) near = block_of(s[u]) >= 0 ? u * NT + tid : near;
            if (near != NONE) atomicMin(&s_near[step & 1], near);       // (a wave may be a step ahead of another's reading)
            __syncthreads();
            const int found = __builtin_amdgcn_readfirstlane(s_near[step & 1]);
            if (found != NONE) {
                row = at + up * found;
                return block_of(p.slots[row]);
            }
        }
        row = -1;
        return -1;
    };
    // the rows that begin a block's run, one a lane: the row before them that has a slot is of another block
    const int slot = slot_of(from + lane), own = block_of(slot), back = block_of(slot_of(from - 1 - lane));
    const uint64_t there = __ballot(from + lane < upto && own >= 0), behind = __ballot(back >= 0);
    if (!there) return;
    int at_row, carry = behind ? __builtin_amdgcn_readlane(back, __builtin_ctzll(behind)) : seek(from - 65, -1, at_row);
    const uint64_t lower = there & ((1ull << lane) - 1);
    const int near = __shfl(own, lower ? 63 - __builtin_clzll(lower) : 0), before = lower ? near : carry;
    uint64_t runs = __ballot((there >> lane & 1) && own != before);
    while (runs) {
        const int at = __builtin_ctzll(runs), first = from + at, blk = __builtin_amdgcn_readlane(own, at);
        const int off0 = __builtin_amdgcn_readlane(slot, at) & (B - 1);
        runs &= runs - 1;
        float *scale = p.scales + ((int64_t)blk * p.n_kv + head) * 2 + which;
        const float was = *scale;
        // How far the run goes (rows without a slot do not end it: a second workgroup would take the same block), and
        // whether it is one row after the other and their slots count up.
        int n = 0;
        bool straight = true;
        for (int at = 0; first + at < p.rows;) {
            const int s = slot_of(first + at + lane), b = block_of(s);
            const uint64_t other = __ballot(b >= 0 && b != blk), ends = other & -other;
            const uint64_t in = __ballot(b == blk) & (ends - 1);     // (no other one: all of them)
            if (in) {
                const int top = 63 - __builtin_clzll(in);
                straight = straight && n == at && in == ~0ull >> (63 - top) &&
                           !__ballot(lane <= top && (s & (B - 1)) != off0 + at + lane);
                n = at + top + 1;
            }
            if (other) break;
            at += 64;
            int row = first + at;
            if (n < at && seek(row, 1, row) != blk) break;
            at = row - first;
        }
        if (!straight) {
            for (int i = tid; i < B; i += NT) s_row[i] = -1;
            __syncthreads();
            for (int i = tid; i < n; i += NT) {
                const int s = p.slots[first + i];
                if (block_of(s) == blk) atomicMax(&s_row[s & (B - 1)], first + i);
            }
            __syncthreads();
        }
        // the tokens that may have rows: m of them from t0 on
        const int t0 = straight ? off0 : 0, m = straight ? n : B;
        auto row_of = [&](int t) { return (unsigned)(t - t0) >= (unsigned)m ? -1 : straight ? first + t - off0 : s_row[t]; };
        const bool anew = row_of(0) >= 0;
        const float held = anew ? 0.f : was;
        uint8_t *store = p.store[which] + ((int64_t)blk * p.n_kv + head) * B * D;
        // item i: of few tokens one after the other, of more sixteen side by side, as the key tiles have them
        const int items = m < 16 ? m * E : (m + 15) / 16 * 16 * E;
        auto token = [&](int i) { return t0 + (m < 16 ? i / E : i / (E * 16) * 16 + (i & 15)); };
        auto group = [&](int i) { return m < 16 ? i % E : i / 16 % E; };
        auto load = [&](int i, float (&v)[16]) {
            const int row = i < items ? row_of(token(i)) : -1;
            if (row < 0) return false;
            const L *from_ = x + row * ld + group(i) * 16;
#pragma unroll
            for (int e = 0; e < 16 / N; ++e) {
                const u32x4 w = *(const typename Piece<L>::raw_t *)(from_ + e * N);
#pragma unroll
                for (int f = 0; f < N; ++f) v[e * N + f] = Piece<L>::get(w, f);
            }
            return true;
        };
        float kept[KEEP][16];
        bool has[KEEP];
        uint32_t top = 0;
        auto largest = [&](const float (&v)[16]) {     // (NaN above infinity above all)
#pragma unroll
            for (int e = 0; e < 16; ++e) top = max(top, __float_as_uint(v[e]) & 0x7FFFFFFFu);
        };
#pragma unroll
        for (int k = 0; k < KEEP; ++k) has[k] = load(tid + k * NT, kept[k]);
#pragma unroll
        for (int k = 0; k < KEEP; ++k)
            if (has[k]) largest(kept[k]);
        for (int i = tid + KEEP * NT; i < items; i += NT) {
            float v[16];
            if (load(i, v)) largest(v);
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
        if (lane == 0) s_top[tid >> 6] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < NT / 64; ++w) top = max(top, s_top[w]);
        const float mine = top >= 0x7F800000u ? __uint_as_float(0x7FC00000u) : __uint_as_float(top) / 127.f;
        float s = __uint_as_float(max(__float_as_uint(mine), __float_as_uint(held) & 0x7FFFFFFFu));
        if (s < 0x1p-126f) s = 0.f;
        const bool finite = __float_as_uint(s) < 0x7F800000u;
        const float inv = finite && s > 0.f ? 1.f / s : 0.f;
        if (tid == 0) *scale = s;
        if (!anew && !(s == held)) {            // what the block holds, to the new scale
            const double inv64 = inv > 0.f ? 1. / (double)s : 0.;
#pragma unroll 1
            for (int i = tid; i < B * E; i += NT) {
                u32x4 w = ((u32x4 *)store)[i];
#pragma unroll 1
                for (int k = 0; k < 4; ++k) {       // (a word at a time, the words in turn: few registers for what is rare)
                    uint32_t r = 0;
#pragma unroll
                    for (int b = 0; b < 4; ++b)
                        r |= (uint32_t)(inv64 > 0. ? round_again((w[0] >> 8 * b) & 255, held, s, inv64) : 128) << 8 * b;
                    w = u32x4{w[1], w[2], w[3], r};
                }
                ((u32x4 *)store)[i] = w;
            }
            __syncthreads();
        }
        auto put = [&](int i, const float (&v)[16]) {
            const u32x4 zero{0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u};
            const u32x4 w = inv > 0.f ? round16(v, s, inv) : zero;
            const int t = token(i);
            if (which == 0) ((u32x4 *)store)[key_piece(t, group(i), D)] = w;
            else *(u32x4 *)(s_stage + (t - t0) * pitch + group(i) * 16) = w;
        };
#pragma unroll
        for (int k = 0; k < KEEP; ++k)
            if (has[k]) put(tid + k * NT, kept[k]);
        for (int i = tid + KEEP * NT; i < items; i += NT) {
            float v[16];
            if (load(i, v)) put(i, v);
        }
        if (which == 1) {
            __syncthreads();
            // the tiles of these tokens; piece i: dimensions e and e + 16, tokens t + v and t + 16 + v
            const int last = (t0 + m - 1) >> 5, pieces = (D >> 5) * 64;
            for (int i = (t0 >> 5) * pieces + tid; i < (last + 1) * pieces; i += NT) {
                const int tile = i >> 6, t = tile / (D >> 5) * 32 + ((i & 63) >> 4) * 4, e = tile % (D >> 5) * 32 + (i & 15);
                uint32_t fresh = 0;
#pragma unroll
                for (int k = 0; k < 8; ++k) fresh |= (uint32_t)(row_of(t + (k >> 2) * 16 + (k & 3)) >= 0) << k;
                if (!fresh) continue;
                u32x4 w{};
                if (fresh != 255) w = ((u32x4 *)store)[i];
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    if (!(fresh >> (k & 7) & 1)) continue;
                    const uint32_t b = s_stage[(t - t0 + ((k >> 2) & 1) * 16 + (k & 3)) * pitch + e + (k >> 3) * 16];
                    w[k >> 2] = (w[k >> 2] & ~(255u << 8 * (k & 3))) | b << 8 * (k & 3);
                }
                ((u32x4 *)store)[i] = w;
            }
        }
        if (runs) __syncthreads();
    }
}

// ---- and back ------------------------------------------------------------------------
template <typename L> struct ReadParams {
    const uint8_t *keys, *values;
    const float *scales;
    const int32_t *slots;
    L *k, *v;
    int rows, blocks, n_kv, D, shift;
};

// A wave reads eight rows of a head: a lane 16 dimensions of a row's keys, and of the
// values, where a token's bytes lie 16 apart, 16 lanes a dimension each of four rows, whose
// bytes are neighbours if their slots are.  8192 rows of 8 heads x 128: 19 us, 2.6 TB/s in and
// out (16 dimensions of a row a thread, bytes apart: 24); storing pairs of dimensions gains nothing.
template <typename L> __global__ __launch_bounds__(256) void k_kv8_read(ReadParams<L> p) {
    constexpr int N = Piece<L>::N;
    const int lane = threadIdx.x & 63, head = blockIdx.y * 4 + (threadIdx.x >> 6), row0 = blockIdx.x * 8;
    if (head >= p.n_kv) return;
    const int B = 1 << p.shift, E = p.D >> 4;
    const int slot = row0 + (lane & 7) < p.rows ? p.slots[row0 + (lane & 7)] : -1;      // (eight lanes a row's)
    const bool there = slot >= 0 && (slot >> p.shift) < p.blocks;
    const int at = there ? slot : 0;
    const int64_t place = (int64_t)(at >> p.shift) * p.n_kv + head;
    float2 scale = make_float2(0.f, 0.f);
    if (there) scale = *(const float2 *)(p.scales + place * 2);
    // keys
    {
        const int i = lane / E, e = lane % E;       // (D = 64: half of the lanes)
        const int64_t b = (((int64_t)__shfl((int)(place >> 32), i & 7) << 32) | (uint32_t)__shfl((int)place, i & 7)) * B * p.D;
        const int t = __shfl(at, i & 7) & (B - 1), ok = __shfl((int)there, i & 7);
        const float s = __shfl(scale.x, i & 7);
        if (i < 8 && row0 + i < p.rows) {
            float k[16];
            u32x4 w{};
            if (ok) w = *((const u32x4 *)(p.keys + b) + key_piece(t, e, p.D));
#pragma unroll
            for (int d = 0; d < 16; ++d) k[d] = ok ? (float)((int)(w[d >> 2] >> 8 * (d & 3) & 255) - 128) * s : 0.f;
            L *to = p.k + (((int64_t)(row0 + i) * p.n_kv + head) * E + e) * 16;
#pragma unroll
            for (int d = 0; d < 16; d += N) *(u32x4 *)(to + d) = Piece<L>::pack(k + d);
        }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int i = 4 * h + (lane >> 4), d = lane & 15;
        const int64_t b = (((int64_t)__shfl((int)(place >> 32), i) << 32) | (uint32_t)__shfl((int)place, i)) * B * p.D;
        const int t = __shfl(at, i) & (B - 1), ok = __shfl((int)there, i);
        const float s = __shfl(scale.y, i);
        if (row0 + i >= p.rows) continue;
        L *to = p.v + ((int64_t)(row0 + i) * p.n_kv + head) * p.D + d;
        const uint8_t *from = p.values + b;
        if (p.D == 128) {
            uint8_t u[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) u[e] = ok ? from[value_byte(t, 16 * e + d, 128)] : 128;
#pragma unroll
            for (int e = 0; e < 8; ++e) Piece<L>::put(to + 16 * e, ok ? (float)((int)u[e] - 128) * s : 0.f);
        } else {
            uint8_t u[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) u[e] = ok ? from[value_byte(t, 16 * e + d, 64)] : 128;
#pragma unroll
            for (int e = 0; e < 4; ++e) Piece<L>::put(to + 16 * e, ok ? (float)((int)u[e] - 128) * s : 0.f);
        }
    }
}

static int log2_of(int n) { return __builtin_ctz((unsigned)n); }

template <typename L, int NT> static bool launch_append(const AppendParams<L> &p, hipStream_t s) {
    const size_t lds = (size_t)(1 << p.shift) * (p.D + 16);
    void *ptrs[] = {(void *)&p};
    return hipLaunchKernel((const void *)k_kv8_append<L, NT>, dim3((p.rows + p.chunk - 1) / p.chunk, p.n_kv, 2), dim3(NT),
                           ptrs, lds, s) == hipSuccess;
}

template <typename L>
static int append(const pipo_kv8 *c, int32_t rows, const L *k, int64_t ld_k, const L *v, int64_t ld_v,
                  const int32_t *d_slots, void *stream) {
    if (!kv8_ok(c) || rows < 0 || rows > kKv8MaxRows) return PIPO_EINVAL;
    if (rows == 0) return PIPO_OK;
    const int64_t least = (int64_t)c->n_kv * c->head_dim;
    if (!kv8_aligned(k, sizeof(L)) || !kv8_aligned(v, sizeof(L)) || !kv8_aligned(d_slots, 4)) return PIPO_EINVAL;
    if (rows > 1 && (ld_k < least || ld_v < least || ld_k > (int64_t)1 << 31 || ld_v > (int64_t)1 << 31)) return PIPO_EINVAL;
    AppendParams<L> p{{k, v}, {ld_k, ld_v}, {c->keys, c->values}, c->scales, d_slots, rows, 1, c->blocks, c->n_kv,
                      c->head_dim, log2_of(c->block)};
    // Rows and threads of a workgroup.  One costs 3 ns whether it finds a block's first row or not, and the runs of one
    // are taken in turn: single tokens want one row a workgroup, prompts a block's.  How long the runs are is not known
    // here.  8 heads x 128, us with 1 / 4 / 16 / 64 rows: 256 single tokens 14 / 19 / 55 / 206 (128 threads; 256: 18 / 17 / 44 /
    // 162), 1024 37 / 40 / 67 / 216, 1000 requests of 5 55 / 43 / 46 / 70, a prompt of 2048 106 / 59 / 22 / 25 (256: 115 /
    // 59 / 20 / 15), of 8192 397 / 202 / 62 / 36 (256: 444 / 218 / 62 / 26; 512: 30).
    const int64_t single = (int64_t)rows * c->n_kv * 2;     // workgroups of one row
    p.chunk = single <= 4096 ? 1 : single >= 64 * 2048 ? 64 : (int)((single + 2047) / 2048);
    hipStream_t s = (hipStream_t)stream;
    const bool ok = single > 1024 && single <= 16384 ? launch_append<L, 128>(p, s) : launch_append<L, 256>(p, s);
    return ok ? PIPO_OK : PIPO_EHIP;
}

template <typename L>
static int read_rows(const pipo_kv8 *c, int32_t rows, const int32_t *d_slots, L *k, L *v, void *stream) {
    if (!kv8_ok(c) || rows < 0 || rows > 64 * kKv8MaxRows) return PIPO_EINVAL;
    if (rows == 0) return PIPO_OK;
    if (!kv8_aligned(d_slots, 4) || !kv8_aligned(k, 16) || !kv8_aligned(v, 16)) return PIPO_EINVAL;
    ReadParams<L> p{c->keys, c->values, c->scales, d_slots, k, v, rows, c->blocks, c->n_kv, c->head_dim, log2_of(c->block)};
    void *ptrs[] = {(void *)&p};
    return hipLaunchKernel((const void *)k_kv8_read<L>, dim3((rows + 7) / 8, (c->n_kv + 3) / 4), dim3(256), ptrs, 0,
                           (hipStream_t)stream) == hipSuccess ? PIPO_OK : PIPO_EHIP;
}

}  // namespace pipo

using namespace pipo;

extern "C" int pipo_kv8_plan(int32_t R, int32_t width, int32_t block, int32_t blocks, const int32_t *d_lens,
                             const int32_t *d_new, int32_t *d_tables, int32_t *d_held, int32_t *d_free,
                             int32_t *d_n_free, int32_t rows, int32_t *d_starts, int32_t *d_total, int32_t *d_slots,
                             int32_t *d_positions, void *stream) {
    if (R < 1 || R > kKv8MaxRows || width < 1 || width > 1 << 20 || blocks < 1 || rows < 0 || rows > kKv8MaxRows) return PIPO_EINVAL;
    if (block != 32 && block != 64 && block != 128 && block != 256) return PIPO_EINVAL;
    if ((int64_t)width * block >= (int64_t)1 << 31 || (int64_t)blocks * block >= (int64_t)1 << 31) return PIPO_EINVAL;
    for (const void *a : {(const void *)d_lens, (const void *)d_new, (const void *)d_tables, (const void *)d_held,
                          (const void *)d_free, (const void *)d_n_free, (const void *)d_starts, (const void *)d_total})
        if (!kv8_aligned(a, 4)) return PIPO_EINVAL;
    if (rows > 0 && (!kv8_aligned(d_slots, 4) || !kv8_aligned(d_positions, 4))) return PIPO_EINVAL;
    PlanParams p{R, width, block, blocks, d_lens, d_new, d_tables, d_held, d_free, d_n_free,
                 rows, d_starts, d_total, d_slots, d_positions, 0};
    hipStream_t s = (hipStream_t)stream;
    p.fill = R <= 1024 && rows <= 4096;
    const bool ok = R <= 256 && rows <= 1024 ? launch(k_kv8_plan<256>, 1, 256, 0, s, p) : launch(k_kv8_plan<1024>, 1, 1024, 0, s, p);
    if (!ok) return PIPO_EHIP;
    if (!p.fill && rows > 0 && !launch(k_kv8_rows, (unsigned)((rows + 255) / 256), 256, 0, s, p)) return PIPO_EHIP;
    return PIPO_OK;
}

extern "C" int pipo_kv8_append(const pipo_kv8 *cache, int32_t rows, const float *d_k, int64_t ld_k, const float *d_v,
                               int64_t ld_v, const int32_t *d_slots, void *stream) {
    return append<float>(cache, rows, d_k, ld_k, d_v, ld_v, d_slots, stream);
}
extern "C" int pipo_kv8_append_bf16(const pipo_kv8 *cache, int32_t rows, const uint16_t *d_k, int64_t ld_k,
                                    const uint16_t *d_v, int64_t ld_v, const int32_t *d_slots, void *stream) {
    return append<uint16_t>(cache, rows, d_k, ld_k, d_v, ld_v, d_slots, stream);
}
extern "C" int pipo_kv8_read(const pipo_kv8 *cache, int32_t rows, const int32_t *d_slots, float *d_k, float *d_v,
                             void *stream) {
    return read_rows<float>(cache, rows, d_slots, d_k, d_v, stream);
}
extern "C" int pipo_kv8_read_bf16(const pipo_kv8 *cache, int32_t rows, const int32_t *d_slots, uint16_t *d_k,
                                  uint16_t *d_v, void *stream) {
    return read_rows<uint16_t>(cache, rows, d_slots, d_k, d_v, stream);
}
