// Keys and values of new tokens into the paged 8-bit cache, positions rotated in on the way, and rows of the cache
// back as floats.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "gala_decode.h"

using namespace gala;

namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 128;      // channels of a block that LDS holds at a time

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

__device__ __forceinline__ int to_code(float x, float inverse) {
    const float t = rintf(x * inverse);
    return t != t ? 0 : (int)fminf(127.0f, fmaxf(-127.0f, t));
}

// One workgroup: the keys or the values of one head in one touched block of one sequence.
template <int TYPE>
__device__ void append_block(const KvArgs &kv, const RopeArgs &rope, const Values &x, int unit, int blocks, float (*tile)[kChunk + 1],
                             float *shared) {
    const int which = unit & 1, h = (unit >> 1) % kv.heads, bj = (unit >> 1) / kv.heads, b = bj / blocks, j = bj % blocks;
    const int start = kv.starts[b], n = kv.starts[b + 1] - start, first = kv.lens[b] - n;
    const int block = max(first, 0) / kKvBlock + j, at = block * kKvBlock;
    const int lo = max(first, at);
    int hi = min(first + min(n, kv.max_new), at + kKvBlock);
    if (which == 0 && rope.table) hi = min(hi, rope.positions);
    if (lo >= hi) return;
    const int page = page_of(kv, b, block);
    if (page < 0) return;
    const int dim = kv.dim, tid = threadIdx.x, count = hi - lo;
    auto value = [&](int t, int d) {
        const long row = start + (lo + t - first);
        auto row_at = [&](int c) { return load_value<TYPE>(x, row, h * dim + c); };
        return which ? row_at(d) : rotated(rope, rope.table + (long)(lo + t) * rope.half * 2, d, row_at);
    };
    // the largest magnitude; chunk by chunk, so that heads of up to 128 channels are loaded once
    float most = 0;
    for (int c0 = 0; c0 < dim; c0 += kChunk) {
        const int cols = min(kChunk, dim - c0);
        for (int e = tid; e < count * cols; e += kThreads) {
            const int t = e / cols, d = e % cols;
            const float v = value(t, c0 + d), a = fabsf(v);
            if (dim <= kChunk) tile[t][d] = v;
            if (a < INFINITY) most = fmaxf(most, a);
        }
    }
    for (int s = 32; s; s >>= 1) most = fmaxf(most, __shfl_xor(most, s));
    if ((tid & 63) == 0) shared[tid >> 6] = most;
    __syncthreads();
    most = fmaxf(fmaxf(shared[0], shared[1]), fmaxf(shared[2], shared[3]));
    float *scale_at = kv.scales + ((long)page * kv.heads + h) * 2 + which;
    const float old = lo > at ? *scale_at : 0.0f;
    __syncthreads();             // every wave has the old scale
    const float scale = fmaxf(old, most * (1.0f / 127.0f)), inverse = scale > 0 ? 1.0f / scale : 0.0f;
    const float rescale = old * inverse;
    const bool grown = lo > at && scale != old;
    if (tid == 0) *scale_at = scale;
    signed char *codes = kv.codes + ((long)page * kv.heads + h) * kv_head_bytes(kv.dim16) + (which ? kKvBlock * 16 * kv.dim16 : 0);
    const int t_lo = lo - at, t_hi = hi - at;
    for (int c0 = 0; c0 < dim; c0 += kChunk) {
        const int cols = min(kChunk, dim - c0);
        if (dim > kChunk) {
            __syncthreads();
            for (int e = tid; e < count * cols; e += kThreads) tile[e / cols][e % cols] = value(e / cols, c0 + e % cols);
            __syncthreads();
        }
        // pieces of 16 codes: keys 16 channels of a token, values 16 tokens of a channel
        const int pieces = 64 * ((cols + 15) / 16);
        for (int i = tid; i < pieces; i += kThreads) {
            const int low = i & 15, mid = (i >> 4) & 3, d16 = i >> 6;     // d16 within the chunk
            const int piece = which ? (c0 / 16 + d16) * 64 + mid * 16 + low : mid * kv.dim16 * 16 + (c0 / 16 + d16) * 16 + low;
            int4 *to = (int4 *)codes + piece;
            signed char c[16];
            bool any = false, all = true;
            for (int k = 0; k < 16; ++k) {
                const int t = which ? (k >> 2) * 16 + mid * 4 + (k & 3) : mid * 16 + low;
                const bool is_new = t >= t_lo && t < t_hi;
                any |= is_new, all &= is_new;
            }
            if (!any && !grown) continue;
            if (!all) *(int4 *)c = *to;
            for (int k = 0; k < 16; ++k) {
                const int t = which ? (k >> 2) * 16 + mid * 4 + (k & 3) : mid * 16 + low;
                const int d = d16 * 16 + (which ? low : k);
                if (t >= t_lo && t < t_hi)
                    c[k] = d < cols ? to_code(tile[t - t_lo][d], inverse) : 0;
                else if (grown)
                    c[k] = (signed char)to_code((float)c[k], rescale);
            }
            *to = *(int4 *)c;
        }
    }
}

// One workgroup: the queries of one token.
template <int TYPE, int OUT>
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
    for (int e = threadIdx.x; e < heads_q * rest; e += kThreads) {
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

// ---- heads of whole 16-byte pieces ---------------------------------------------------------------------------------
// A thread takes pieces of eight channels of a token, in the half layout both members of eight pairs.  Four
// neighbouring lanes have the same channels of four tokens of a row, so that loads are whole lines of four rows and
// the values' codes, which lie token by token, are put together by an exchange within the four lanes.

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

// Of four lanes' words the bytes of the lane's number: lane r gets byte r of lanes 0, 1, 2 and 3.
__device__ __forceinline__ u32 quad_transpose(u32 w) {
    const u32 a = __builtin_amdgcn_mov_dpp(w, 0x00, 0xf, 0xf, true), b = __builtin_amdgcn_mov_dpp(w, 0x55, 0xf, 0xf, true);
    const u32 c = __builtin_amdgcn_mov_dpp(w, 0xaa, 0xf, 0xf, true), d = __builtin_amdgcn_mov_dpp(w, 0xff, 0xf, 0xf, true);
    const u32 pick = 0x0c0c0400u + 0x0101u * (threadIdx.x & 3);
    return __builtin_amdgcn_perm(b, a, pick) | __builtin_amdgcn_perm(d, c, pick) << 16;
}
// four codes in a word
__device__ __forceinline__ u32 codes_of(const float *x, float inverse) {
    u32 w = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) w |= (u32)(to_code(x[k], inverse) & 255) << 8 * k;
    return w;
}
// offsets of the codes of channels d .. d+7 of token t: of keys they lie together, of values 16 bytes apart
__device__ __forceinline__ int key_place(int t, int d, int dim16) { return ((t >> 4) * dim16 + (d >> 4)) * 256 + (t & 15) * 16 + (d & 15); }
__device__ __forceinline__ int value_place(int t, int d) { return (d >> 4) * 1024 + ((t & 15) >> 2) * 256 + (d & 15) * 16 + (t >> 4) * 4 + (t & 3); }

// One workgroup: the keys or the values of one head in one touched block of one sequence, as many new tokens as
// THREADS / 4.  The values wait in registers for the block's scale.
template <int TYPE, int THREADS, int MOST16>
__device__ void append_pieces(const KvArgs &kv, const RopeArgs &rope, const Values &x, const Pieces &pieces, int which, int h, int b, int j,
                              signed char *tile, float *shared) {
    // Items a thread may have of each kind, and rows of registers for both: pairs take rows from the front, singles from the
    // back.  With p pairs of m x 16 channels that is 2 ceil(p / 4) + ceil((m - p) / 2), at most m / 2 + 2.
    constexpr int kTokens = THREADS / 4, kPairs = (MOST16 * kTokens + THREADS - 1) / THREADS, kSingles = (2 * MOST16 * kTokens + THREADS - 1) / THREADS;
    constexpr int kRows = MOST16 / 2 + 2;
    const int start = kv.starts[b], n = kv.starts[b + 1] - start, first = kv.lens[b] - n;
    const int block = max(first, 0) / kKvBlock + j, at = block * kKvBlock;
    const int lo = max(first, at);
    int hi = min(first + min(n, kv.max_new), at + kKvBlock);
    if (which == 0 && rope.table) hi = min(hi, rope.positions);
    if (lo >= hi) return;
    const int page = page_of(kv, b, block);
    if (page < 0) return;
    const int dim = kv.dim, tid = threadIdx.x, count = hi - lo;
    float *scale_at = kv.scales + ((long)page * kv.heads + h) * 2 + which;
    const float old = lo > at ? *scale_at : 0.0f;
    const int pairs = which ? 0 : pieces.pairs, singles = which ? kv.dim16 * 2 : pieces.singles;
    const Divisor of_singles = which ? Divisor(kv.dim16 * 2) : pieces.of_singles;
    float v[kRows][8], most = 0;
    // item q of a token's pieces: lane r of four has token 4 * quad + r
    auto token_of = [&](int q, const Divisor &of, int &piece) {
        const int rest = q >> 2, quad = of(rest);
        piece = rest - quad * of.d;
        return quad * 4 + (q & 3);
    };
    auto meet = [&](const float (&row)[8]) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float a = fabsf(row[k]);
            if (a < INFINITY) most = fmaxf(most, a);
        }
    };
#pragma unroll
    for (int k = 0; k < kPairs; ++k) {
        int piece;
        const int q = tid + k * THREADS, t = token_of(q, pieces.of_pairs, piece);
        if (pairs && t < count) {
            const long row = start + (lo + t - first);
            load_piece<TYPE>(x, row, h * dim + piece * 8, v[2 * k]);
            load_piece<TYPE>(x, row, h * dim + rope.half + piece * 8, v[2 * k + 1]);
            turn(rope.table + ((long)(lo + t) * rope.half + piece * 8) * 2, v[2 * k], v[2 * k + 1]);
            meet(v[2 * k]), meet(v[2 * k + 1]);
        }
    }
#pragma unroll
    for (int k = 0; k < kSingles; ++k) {
        int piece;
        const int q = tid + k * THREADS, t = token_of(q, of_singles, piece), d = (2 * pairs + piece) * 8;
        float (&own)[8] = v[kRows - 1 - k];
        if (singles && t < count) {
            if (d < dim) {
                load_piece<TYPE>(x, start + (lo + t - first), h * dim + d, own);
                if (!which && rope.table && rope.interleaved && d < 2 * rope.half) turn(rope.table + ((long)(lo + t) * rope.half + d / 2) * 2, own);
                meet(own);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) own[i] = 0;
            }
        }
    }
    for (int k = 32; k; k >>= 1) most = fmaxf(most, __shfl_xor(most, k));
    if ((tid & 63) == 0) shared[tid >> 6] = most;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < THREADS / 64; ++k) most = fmaxf(most, shared[k]);
    const float scale = fmaxf(old, most * (1.0f / 127.0f)), inverse = scale > 0 ? 1.0f / scale : 0.0f;
    if (tid == 0) *scale_at = scale;              // every wavefront has waited for the old one
    signed char *codes = kv.codes + ((long)page * kv.heads + h) * kv_head_bytes(kv.dim16) + (which ? kKvBlock * 16 * kv.dim16 : 0);
    const int t_lo = lo - at;
    const bool whole = count == kKvBlock;
    if (lo > at && scale != old) {
        const float rescale = old * inverse;
        for (int i = tid; i < kv.dim16 * 64; i += THREADS) {
            union {
                int4 word;
                signed char c[16];
            } u;
            u.word = ((int4 *)codes)[i];
#pragma unroll
            for (int k = 0; k < 16; ++k) u.c[k] = (signed char)to_code((float)u.c[k], rescale);
            ((int4 *)codes)[i] = u.word;
        }
        __syncthreads();
    }
    // a whole block is put in order in LDS, part of one goes to its places
    auto put = [&](int t, int d, const float (&row)[8]) {
        const u32 low = codes_of(row, inverse), high = codes_of(row + 4, inverse);
        if (which == 0) {
            *(uint2 *)((whole ? tile : codes) + key_place(t, d, kv.dim16)) = uint2{low, high};
        } else if (whole) {
            u32 *to = (u32 *)(tile + value_place(t & ~3, d) + (t & 3) * 16);
            to[0] = quad_transpose(low), to[16] = quad_transpose(high);
        } else {
            signed char *to = codes + value_place(t, d);
#pragma unroll
            for (int k = 0; k < 4; ++k) to[16 * k] = (signed char)(low >> 8 * k), to[16 * (k + 4)] = (signed char)(high >> 8 * k);
        }
    };
#pragma unroll
    for (int k = 0; k < kPairs; ++k) {
        int piece;
        const int q = tid + k * THREADS, t = token_of(q, pieces.of_pairs, piece);
        if (pairs && t < count) put(t_lo + t, piece * 8, v[2 * k]), put(t_lo + t, rope.half + piece * 8, v[2 * k + 1]);
    }
#pragma unroll
    for (int k = 0; k < kSingles; ++k) {
        int piece;
        const int q = tid + k * THREADS, t = token_of(q, of_singles, piece), d = (2 * pairs + piece) * 8;
        if (singles && t < count) put(t_lo + t, d, v[kRows - 1 - k]);
    }
    if (whole) {
        __syncthreads();
        for (int i = tid; i < kv.dim16 * 64; i += THREADS) ((int4 *)codes)[i] = ((int4 *)tile)[i];
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

// Workgroups of a launch: `units` with a block each, then those with `tokens` tokens' queries each, `rows` of a sequence.
struct Shares {
    Order order;
    int blocks, groups, tokens, rows;
};

// x' = turn by the position's angle, scale = max(scale, max|x'| / 127), code = rint(x' / scale).  A workgroup has a whole block
// of a head, so that the scale it needs is found and used in one launch and the rows are read once.  Bound by HBM in
// prompts (4 x 2000 tokens of 24 heads of 128 residues: 214 MB in 57 us with the export, 3.8 TB/s) and by its chain of loads
// for single tokens (starts, table, row, scale: 5 us).
template <int TYPE, int OUT, int THREADS, int MOST16>
__global__ __launch_bounds__(THREADS) void kv_append_kernel(KvArgs kv, RopeArgs rope, int heads_q, Values q, Values q_out, Values k, Values v,
                                                            Shares shares) {
    __shared__ alignas(16) signed char tile[THREADS == 256 ? kKvBlock * 16 * MOST16 : 16];
    __shared__ float shared[THREADS / 64];
    if ((int)blockIdx.x < shares.groups) {
        const int2 unit = shares.order.unit_of(blockIdx.x);
        if (unit.x >= shares.order.blocks) return;
        const int which = unit.y & 1, h = unit.y >> 1, b = unit.x / shares.blocks;
        append_pieces<TYPE, THREADS, MOST16>(kv, rope, which ? v : k, Pieces(16 * kv.dim16, rope.half, rope.interleaved), which, h, b,
                                             unit.x - b * shares.blocks, tile, shared);
    } else {
        const int u = blockIdx.x - shares.groups, b = u / shares.rows;
        rotate_pieces<TYPE, OUT, THREADS>(kv, rope, q, q_out, Pieces(kv.dim, rope.half, rope.interleaved), heads_q, b,
                                          (u - b * shares.rows) * shares.tokens, shares.tokens);
    }
}
// The same for rows of any size and place, number by number: 2000 tokens of 24 + 2 x 24 heads of 80 bf16 channels take
// 65 us with the export that follows them, and 23 us in pieces; one token of 64 sequences 34 us and 13 us.
template <int TYPE, int OUT>
__global__ __launch_bounds__(kThreads) void kv_append_any_kernel(KvArgs kv, RopeArgs rope, int heads_q, Values q, Values q_out, Values k,
                                                                 Values v, int blocks, int units) {
    __shared__ float tile[kKvBlock][kChunk + 1];
    __shared__ float shared[4];
    const int unit = blockIdx.x;
    if (unit < units)
        append_block<TYPE>(kv, rope, unit & 1 ? v : k, unit, blocks, tile, shared);
    else
        rotate_row<TYPE, OUT>(kv, rope, q, q_out, heads_q, unit - units);
}

// One workgroup: the keys or the values of one head in one block of one sequence, through LDS where rows are in pieces.  Bound by
// HBM (8191 tokens of 48 heads of 80 f16 values: 94 MB in 19 us).
template <int OUT, bool PIECES>
__global__ __launch_bounds__(kThreads) void kv_export_kernel(KvArgs kv, Values k_out, Values v_out, int blocks, Order order) {
    const int2 unit = order.unit_of(blockIdx.x);
    if (unit.x >= order.blocks) return;
    const int which = unit.y & 1, h = unit.y >> 1, b = unit.x / blocks, j = unit.x - b * blocks;
    const int start = kv.starts[b], n = kv.starts[b + 1] - start, first = kv.lens[b] - n;
    // tokens at negative positions are in blocks of their own numbers, down from -1
    const int block = (first >= 0 ? first / kKvBlock : -((63 - first) / kKvBlock)) + j, at = block * kKvBlock;
    const int lo = max(first, at), hi = min(first + min(n, kv.max_new), at + kKvBlock);
    if (lo >= hi) return;
    const int page = page_of(kv, b, block);
    const Values &out = which ? v_out : k_out;
    const float scale = page < 0 ? 0.0f : kv.scales[((long)page * kv.heads + h) * 2 + which];
    const signed char *codes = page < 0 ? nullptr : kv.codes + ((long)page * kv.heads + h) * kv_head_bytes(kv.dim16) + (which ? kKvBlock * 16 * kv.dim16 : 0);
    const int tid = threadIdx.x;
    if constexpr (PIECES) {
        __shared__ alignas(16) signed char tile[kKvBlock * kMaxHeadDim];
        if (page >= 0)
            for (int i = tid; i < kv.dim16 * 64; i += kThreads) ((int4 *)tile)[i] = ((const int4 *)codes)[i];
        __syncthreads();
        const Divisor of(kv.dim / 8);
        const int quad0 = (lo - at) >> 2, quads = ((hi - at + 3) >> 2) - quad0;
        for (int q = tid; q < quads * 4 * kv.dim / 8; q += kThreads) {          // whole quads of lanes
            const int rest = q >> 2, quad = of(rest), d = (rest - quad * (int)of.d) * 8, t = (quad0 + quad) * 4 + (q & 3);
            u32 low = 0, high = 0;
            if (page >= 0) {
                if (which) {
                    const u32 *from = (const u32 *)(tile + value_place(t & ~3, d) + (t & 3) * 16);
                    low = quad_transpose(from[0]), high = quad_transpose(from[16]);
                } else {
                    const uint2 both = *(const uint2 *)(tile + key_place(t, d, kv.dim16));
                    low = both.x, high = both.y;
                }
            }
            if (t < lo - at || t >= hi - at) continue;
            float x[8];
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = (float)(signed char)(low >> 8 * k) * scale, x[4 + k] = (float)(signed char)(high >> 8 * k) * scale;
            if (page < 0) {
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] = 0;
            }
            store_piece<OUT>(out, start + (at + t - first), h * kv.dim + d, x);
        }
    } else {
        for (int e = tid; e < (hi - lo) * kv.dim; e += kThreads) {
            const int t = lo - at + e / kv.dim, d = e % kv.dim;
            const int place = which ? value_place(t, d) : key_place(t, d, kv.dim16);
            const float x = page < 0 ? 0.0f : (float)codes[place] * scale;
            store_value<OUT>(out, start + (at + t - first), h * kv.dim + d, x);
        }
    }
}

// whether every piece of eight channels of every row lies on 16 bytes
bool in_pieces(const Values &v, int dim) {
    const size_t size = v.type == GALA_F32 ? 4 : v.type == GALA_RESIDUE ? 8 : 2;
    return !v.data || ((uintptr_t)v.data % 16 == 0 && v.stride * size % 16 == 0 && dim % 8 == 0);
}

}  // namespace

namespace gala {

int launch_kv_append(void *stream, const KvArgs &kv, const RopeArgs &rope, int heads_q, const Values &q, const Values &q_out,
                     const Values &k, const Values &v) {
    // the most blocks that max_new tokens in a row can touch
    const int blocks = (kv.max_new + kKvBlock - 2) / kKvBlock + 1, units = k.data ? kv.count * blocks * kv.heads * 2 : 0;
    const int rows = heads_q ? kv.count * kv.max_new : 0;
    hipStream_t st = (hipStream_t)stream;
    // pairs in pieces too: halves of eight channels, and interleaved channels of four pairs
    const bool pieces = in_pieces(q, kv.dim) && in_pieces(q_out, kv.dim) && in_pieces(k, kv.dim) && in_pieces(v, kv.dim) &&
                        (!rope.table || ((uintptr_t)rope.table % 16 == 0 && rope.half % (rope.interleaved ? 4 : 8) == 0)) &&
                        (long)heads_q * kv.dim / 8 < 65536;
    by_type(k.data ? k.type : q.type, [&](auto type) {
        by_type(q_out.type, [&](auto out) {
            constexpr int T = decltype(type)::value, O = decltype(out)::value;
            if constexpr (O != GALA_RESIDUE) {
                if (!pieces) {
                    hipLaunchKernelGGL((kv_append_any_kernel<T, O>), dim3(units + rows), dim3(kThreads), 0, st, kv, rope, heads_q, q, q_out,
                                       k, v, blocks, units);
                    return;
                }
                auto launch = [&](auto threads, auto most16) {
                    constexpr int N = decltype(threads)::value, M = decltype(most16)::value;
                    // two items a thread, where a sequence has as many
                    const int items = std::max(1, heads_q * kv.dim / 16);
                    Shares s{order_of(k.data ? kv.count * blocks : 0, kv.heads, kv.dim, k), blocks, 0, std::max(1, std::min(2 * N / items, kv.max_new)), 0};
                    s.groups = s.order.groups();
                    s.rows = (kv.max_new + s.tokens - 1) / s.tokens;
                    hipLaunchKernelGGL((kv_append_kernel<T, O, N, M>), dim3(s.groups + (heads_q ? kv.count * s.rows : 0)), dim3(N), 0, st, kv, rope,
                                       heads_q, q, q_out, k, v, s);
                };
                // A few tokens need a wavefront, many a block's worth: 4 tokens of 256 sequences take 36 us with the export so and 51 us
                // in workgroups of 256, 16 tokens 65 and 73.  Heads of up to 128 channels have half the registers.
                const bool few = kv.max_new <= 16, narrow = kv.dim16 <= 8;
                if (few && narrow) launch(std::integral_constant<int, 64>(), std::integral_constant<int, 8>());
                if (few && !narrow) launch(std::integral_constant<int, 64>(), std::integral_constant<int, 16>());
                if (!few && narrow) launch(std::integral_constant<int, 256>(), std::integral_constant<int, 8>());
                if (!few && !narrow) launch(std::integral_constant<int, 256>(), std::integral_constant<int, 16>());
            }
        });
    });
    return hipGetLastError() != hipSuccess;
}

int launch_kv_export(void *stream, const KvArgs &kv, const Values &k_out, const Values &v_out) {
    const int blocks = (kv.max_new + kKvBlock - 2) / kKvBlock + 1;
    const Order order = order_of(kv.count * blocks, kv.heads, kv.dim, k_out);
    const dim3 grid(order.groups());
    by_type(k_out.type, [&](auto type) {
        constexpr int T = decltype(type)::value;
        if (in_pieces(k_out, kv.dim) && in_pieces(v_out, kv.dim))
            hipLaunchKernelGGL((kv_export_kernel<T, true>), grid, dim3(kThreads), 0, (hipStream_t)stream, kv, k_out, v_out, blocks, order);
        else
            hipLaunchKernelGGL((kv_export_kernel<T, false>), grid, dim3(kThreads), 0, (hipStream_t)stream, kv, k_out, v_out, blocks, order);
    });
    return hipGetLastError() != hipSuccess;
}

}  // namespace gala
