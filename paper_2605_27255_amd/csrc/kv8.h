// The paged 8-bit cache of the serving operators: where a block's bytes lie, and
// the rounding to them.
#pragma once
#include "opd_rows.h"
#include "pipo.h"

namespace pipo {

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;

constexpr int kKv8MaxRows = 1 << 20;
// (checks on the host)
bool kv8_ok(const pipo_kv8 *c);
inline bool kv8_aligned(const void *p, size_t to) { return p && ((uintptr_t)p & (to - 1)) == 0; }

// A piece of 16 bytes is what a lane of a wave feeds to two MFMAs, so that a wave's
// 16-byte load of a tile is one contiguous 1 KB read: of a 16-token key tile lane
// 16 g + r holds token r, dimensions 16 g .. 16 g + 15 of 64 (the products may
// take a dot product's terms in any order, and the queries are loaded alike); of
// a 32-token value tile it holds dimensions r and 16 + r of 32, of each the eight
// tokens 4 g + v and 16 + 4 g + v, whose probabilities the lanes of group g hold.
__device__ __forceinline__ int key_piece(int t, int e16, int D) {      // e16: dimension / 16
    return ((t >> 4) * (D >> 6) + (e16 >> 2)) * 64 + (e16 & 3) * 16 + (t & 15);
}
__device__ __forceinline__ int value_byte(int t, int e, int D) {
    return (((t >> 5) * (D >> 5) + (e >> 5)) * 64 + ((t & 15) >> 2) * 16 + (e & 15)) * 16 + (e & 16) / 2 +
           ((t & 16) >> 2) + (t & 3);
}

// A request's rows first .. first + n - 1 from the two starts around them, whatever these hold: both are cut off to
// the call's rows before anything is computed with them, so that no difference or product passes 32 bits.
struct RequestRows { int first, n; };
__host__ __device__ __forceinline__ RequestRows request_rows(int32_t from, int32_t to, int32_t rows) {
    const int a = from < 0 ? 0 : from < rows ? from : rows, b = to < rows ? to : rows;
    return RequestRows{a, b > a ? b - a : 0};
}

// Request of a row: the last r with starts[r] <= row (0 <= r < R), the row not before starts[0].
__device__ __forceinline__ int request_of(const int32_t *starts, int R, int row) {
    int lo = 0, hi = R;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (starts[mid] <= row) lo = mid; else hi = mid;
    }
    return lo;
}

}  // namespace pipo
