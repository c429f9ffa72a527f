// Rows of heads, number by number or in pieces of eight channels: how they are read and written, and positions rotated into
// them.  For the kernels that bring keys, values and queries into a cache or on their way to one.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "gala_decode.h"

namespace gala {
namespace {

// Channel d of a row with its position rotated in; row_at(d) gives the row's channels, table the position's angles.
// Products and sums are rounded one by one: a code that falls on the edge between two is then the same for everybody
// who rotates in 32 bits.
template <class F>
__device__ __forceinline__ float rotated(const RopeArgs &r, const float *table, int d, F row_at) {
#pragma clang fp contract(off)
    const float x = row_at(d);
    if (d >= 2 * r.half || !r.table) return x;
    const bool second = r.interleaved ? d & 1 : d >= r.half;
    const int i = r.interleaved ? d >> 1 : second ? d - r.half : d;
    const float other = row_at(r.interleaved ? d ^ 1 : second ? d - r.half : d + r.half);
    const float c = table[2 * i] * x, s = table[2 * i + 1] * other;
    return second ? c + s : c - s;
}

// n / d for n and d below 2^16
struct Divisor {
    u32 d, inverse;
    __host__ __device__ explicit Divisor(u32 d) : d(d), inverse(0xffffffffu / d + 1) {}
    __device__ u32 operator()(u32 n) const { return d == 1 ? n : __umulhi(n, inverse); }
};

// How a head's channels fall into pieces: `pairs` pieces that have a partner, then `singles` without.
struct Pieces {
    int pairs, singles;
    Divisor of_pairs, of_singles;
    __host__ __device__ Pieces(int channels, int half, bool interleaved)
        : pairs(interleaved ? 0 : half / 8), singles(channels / 8 - 2 * pairs), of_pairs(pairs > 0 ? pairs : 1), of_singles(singles > 0 ? singles : 1) {}
};

template <int TYPE>
__device__ __forceinline__ void load_piece(const Values &v, long row, int column, float (&x)[8]) {
    typedef typename Element<TYPE>::type E;
    union {
        int4 word[sizeof(E) / 2];
        E e[8];
    } u;
    const int4 *from = (const int4 *)((const E *)v.data + row * v.stride + column);
#pragma unroll
    for (int k = 0; k < (int)sizeof(E) / 2; ++k) u.word[k] = from[k];
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = to_float<TYPE>(u.e[k], v.unit, v.p);
}
template <int TYPE>
__device__ __forceinline__ void store_piece(const Values &v, long row, int column, const float (&x)[8]) {
    typedef typename Element<TYPE>::type E;
    union {
        int4 word[sizeof(E) / 2];
        E e[8];
    } u;
#pragma unroll
    for (int k = 0; k < 8; ++k) u.e[k] = from_float<TYPE>(x[k], v.unit, v.p);
    int4 *to = (int4 *)((E *)v.data + row * v.stride + column);
#pragma unroll
    for (int k = 0; k < (int)sizeof(E) / 2; ++k) to[k] = u.word[k];
}
// as in rotated(): products and sums rounded one by one
__device__ __forceinline__ void turn(const float *table, float (&a)[8], float (&b)[8]) {
#pragma clang fp contract(off)
    float t[16];
#pragma unroll
    for (int k = 0; k < 4; ++k) *(float4 *)(t + 4 * k) = ((const float4 *)table)[k];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const float x = a[k], y = b[k], c = t[2 * k], s = t[2 * k + 1];
        a[k] = c * x - s * y;
        b[k] = c * y + s * x;
    }
}
__device__ __forceinline__ void turn(const float *table, float (&a)[8]) {
#pragma clang fp contract(off)
    float t[8];
#pragma unroll
    for (int k = 0; k < 2; ++k) *(float4 *)(t + 4 * k) = ((const float4 *)table)[k];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float x = a[2 * k], y = a[2 * k + 1], c = t[2 * k], s = t[2 * k + 1];
        a[2 * k] = c * x - s * y;
        a[2 * k + 1] = c * y + s * x;
    }
}

// One workgroup: the queries of one token.
template <int TYPE, int OUT, int THREADS>
__device__ void rotate_row(const KvArgs &kv, const RopeArgs &rope, const Values &q, const Values &q_out, int heads_q, int unit) {
    const int b = unit / kv.max_new, i = unit % kv.max_new;
    const int start = kv.starts[b], n = kv.starts[b + 1] - start;
    if (i >= n) return;
    const int t = kv.lens[b] - n + i, dim = kv.dim;
    const bool has = !rope.table || (t >= 0 && t < rope.positions);
    const float *table = rope.table && has ? rope.table + (long)t * rope.half * 2 : nullptr;
    const long row = start + i;
    // a pair by one thread, so that q_out may be q
    const int half = rope.table ? rope.half : 0, rest = dim - half;
    for (int e = threadIdx.x; e < heads_q * rest; e += THREADS) {
        const int h = e / rest, k = e % rest;
        auto row_at = [&](int c) { return load_value<TYPE>(q, row, h * dim + c); };
        if (k < half) {
            const int d0 = rope.interleaved ? 2 * k : k, d1 = rope.interleaved ? 2 * k + 1 : k + half;
            float x = __builtin_nanf(""), y = x;
            if (has) x = rotated(rope, table, d0, row_at), y = rotated(rope, table, d1, row_at);
            store_value<OUT>(q_out, row, h * dim + d0, x);
            store_value<OUT>(q_out, row, h * dim + d1, y);
        } else {
            store_value<OUT>(q_out, row, h * dim + half + k, has ? row_at(half + k) : __builtin_nanf(""));
        }
    }
}

// One workgroup: the queries of a few tokens.
template <int TYPE, int OUT, int THREADS>
__device__ void rotate_pieces(const KvArgs &kv, const RopeArgs &rope, const Values &q, const Values &q_out, const Pieces &pieces, int heads_q,
                              int b, int i0, int tokens) {
    const int start = kv.starts[b], n = kv.starts[b + 1] - start, first = kv.lens[b] - n, dim = kv.dim;
    tokens = min(tokens, min(n, kv.max_new) - i0);
    const int each = pieces.pairs + pieces.singles;
    const Divisor of_each(each), of_heads(heads_q);
    for (int e = threadIdx.x; e < tokens * heads_q * each; e += THREADS) {
        const int rest = of_each(e), piece = e - rest * each, i = i0 + of_heads(rest), h = rest - (i - i0) * heads_q;
        const int t = first + i;
        const bool has = !rope.table || (t >= 0 && t < rope.positions);
        const long row = start + i;
        float x[8], y[8];
        if (piece < pieces.pairs) {
            const int d = piece * 8;
            load_piece<TYPE>(q, row, h * dim + d, x);
            load_piece<TYPE>(q, row, h * dim + rope.half + d, y);
            if (has) {
                turn(rope.table + ((long)t * rope.half + d) * 2, x, y);
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] = y[k] = __builtin_nanf("");
            }
            store_piece<OUT>(q_out, row, h * dim + d, x);
            store_piece<OUT>(q_out, row, h * dim + rope.half + d, y);
        } else {
            const int d = (pieces.pairs + piece) * 8;
            load_piece<TYPE>(q, row, h * dim + d, x);
            if (has && rope.table && rope.interleaved && d < 2 * rope.half) turn(rope.table + ((long)t * rope.half + d / 2) * 2, x);
            if (!has) {
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] = __builtin_nanf("");
            }
            store_piece<OUT>(q_out, row, h * dim + d, x);
        }
    }
}

// products and sums rounded one by one
__device__ __forceinline__ void turn_pair(float cos, float sin, float &x, float &y) {
#pragma clang fp contract(off)
    const float a = cos * x - sin * y, b = cos * y + sin * x;
    x = a, y = b;
}
// How a workgroup turns rows of heads: threads take a piece of a row, in the half layout both members of eight pairs, find its angles
// once and turn it in every `slots`-th head.
struct Turns {
    Pieces pieces;
    int half, heads, dim, slots;
    int rows, parts;                         // rows of a workgroup, or workgroups of a row
};
inline Turns turns_of(long rows, int heads, int dim, int half, bool interleaved, int threads) {
    const Pieces pieces(dim, half, interleaved);
    const int each = std::max(1, pieces.pairs + pieces.singles);         // none in rows of less than a piece
    // One head a thread where that does not fill the card twice: 6000 rows of 32 heads of 128 bf16 channels take 25.1 us with one, 22.7 with
    // two, 23.5 with four.
    const long turns = std::min(2l, std::max(1l, rows * each * heads / (256 * 512)));
    int slots = (int)((heads + turns - 1) / turns);
    slots = std::min(slots, std::max(1, 32768 / each));
    return Turns{pieces, half, heads, dim, slots, std::max(1, threads / (each * slots)), (each * slots + threads - 1) / threads};
}
// part: of the row, where it has several workgroups; row_of(r): row r of the workgroup's, -1 for none; angles(row, two, d, angle): the angles of the piece at channel d, whether there are any
template <int TYPE, int OUT, int THREADS, class R, class A>
__device__ __forceinline__ void turn_heads(const Turns &t, int part, const Values &x, const Values &out, R row_of, A angles) {
    const int pairs = t.pieces.pairs, each = pairs + t.pieces.singles, slots = t.slots, heads = t.heads, dim = t.dim, half = t.half;
    const int e = part * THREADS + threadIdx.x;
    const Divisor of_row(each * slots), of_each(each);
    if (e < t.rows * each * slots) {
        const int r = of_row(e), rest = e - r * each * slots, slot = of_each(rest), piece = rest - slot * each;
        const long row = row_of(r);
        if (row < 0) return;
        const bool two = piece < pairs;
        const int d = two ? piece * 8 : (pairs + piece) * 8;          // singles lie behind both members of the pairs
        const bool turned = d < 2 * half;
        float angle[16] = {};                    // cosine and sine of each pair
        const bool has = angles(r, two, turned, d, angle);
        // one head at a time: two under way take registers from other wavefronts (25.4 us against 22.7 for the rows above)
        for (int h = slot; h < heads; h += slots) {
            float u[8], v[8] = {};
            load_piece<TYPE>(x, row, h * dim + d, u);
            if (two) load_piece<TYPE>(x, row, h * dim + half + d, v);
            if (turned && two) {
#pragma unroll
                for (int k = 0; k < 8; ++k) turn_pair(angle[2 * k], angle[2 * k + 1], u[k], v[k]);
            } else if (turned) {
#pragma unroll
                for (int k = 0; k < 4; ++k) turn_pair(angle[2 * k], angle[2 * k + 1], u[2 * k], u[2 * k + 1]);
            }
            if (!has) {
#pragma unroll
                for (int k = 0; k < 8; ++k) u[k] = v[k] = __builtin_nanf("");
            }
            store_piece<OUT>(out, row, h * dim + d, u);
            if (two) store_piece<OUT>(out, row, h * dim + half + d, v);
        }
    }
}

// The order of a launch's workgroups with a block of a head each.  Workgroups go to the eight XCDs in turn; where a head's
// part of a row does not end on a cache line, neighbouring heads share lines, and all heads of a block go to one XCD.  8191
// tokens of 72 heads of 80 f16 channels take 84 us so, with the export that follows them, and 90 us in turn; whole lines gain nothing
// (4 x 2000 tokens of 128 channels 57 us in turn).
struct Order {
    int blocks, heads;       // blocks of all sequences; twice the heads: keys and values
    bool together;
    __host__ __device__ int groups() const { return (together ? (blocks + 7) / 8 * 8 : blocks) * heads; }
    // (block, 2 head + which); no such block: nothing to do
    __device__ int2 unit_of(int group) const {
        if (!together) return int2{group / heads, group % heads};
        const int in_xcd = group >> 3, row = in_xcd / heads;
        return int2{row * 8 + (group & 7), in_xcd - row * heads};
    }
};
Order order_of(int blocks, int heads, int dim, const Values &v) {
    const int size = v.type == GALA_F32 ? 4 : v.type == GALA_RESIDUE ? 8 : 2;
    // padding rounds the blocks up to eight
    return Order{blocks, 2 * heads, dim * size % 128 != 0 && blocks >= 32};
}

// whether every piece of eight channels of every row lies on 16 bytes
bool in_pieces(const Values &v, int dim) {
    const size_t size = v.type == GALA_F32 ? 4 : v.type == GALA_RESIDUE ? 8 : 2;
    return !v.data || ((uintptr_t)v.data % 16 == 0 && v.stride * size % 16 == 0 && dim % 8 == 0);
}

}  // namespace
}  // namespace gala
