// Attention of a batch's queries over the paged 8-bit cache.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "gala_decode.h"

using namespace gala;

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));

constexpr int kColumns = 16;         // queries that a wavefront's products take at once
constexpr float kLog2E = 1.4426950408889634f;

struct Attention {
    KvArgs kv;
    Values q, out;
    bool pieces, out_quads;          // rows of q lie on 16 bytes, those of out on four values
    int heads_q, group;              // group: query heads of a head of the cache
    float scale;
    int window, sinks;
    int waves;                       // wavefronts of a workgroup
    int tiles, splits, columns;      // column tiles of a head, shares of its keys, columns of a tile that are kept
    float *sums, *stats;             // of every share: columns x dim, and columns x (largest, sum)
};

// The blocks that the queries of one column tile see: the first tokens', then the window's.
struct Seen {
    int start, n, col0, cols;        // first row, rows, first column and columns of the tile
    int at_lo, at_hi;                // positions of the tile's queries
    int first, begin, total;         // first: blocks of first tokens in front of `begin`

    __device__ int block(int u) const { return u < first ? u : begin + (u - first); }
};
__device__ __forceinline__ Seen seen_by(const Attention &a, int b, int tile, int columns = kColumns) {
    Seen s;
    s.start = a.kv.starts[b];
    const int all = a.kv.starts[b + 1] - s.start, len = a.kv.lens[b];
    s.n = min(all, a.kv.max_new);
    s.col0 = tile * columns;
    s.cols = max(0, min(columns, s.n * a.group - s.col0));
    s.at_lo = len - all + s.col0 / a.group;
    s.at_hi = len - all + (s.col0 + max(s.cols, 1) - 1) / a.group;
    const int end = min(s.at_hi + 1, min(a.kv.max_len, a.kv.table_stride * kKvBlock));       // keys from here on are not seen
    const int last = end > 0 ? (end + kKvBlock - 1) / kKvBlock : 0;
    s.begin = a.window ? min(max(0, s.at_lo - a.window + 1) / kKvBlock, last) : 0;
    s.first = min((int)min((long)a.sinks + kKvBlock - 1, 0x7fffffffl) / kKvBlock, s.begin);
    s.total = s.cols && a.kv.pages ? s.first + last - s.begin : 0;
    return s;
}
// blocks of a share
__device__ __forceinline__ int share_of(const Attention &a, int total) {
    const int each = (total + a.splits - 1) / a.splits;
    return (each + a.waves - 1) / a.waves * a.waves;
}

// 8 x N channels of a row from `column` on, 0 from `end` on; eight at a load where rows lie on 16 bytes
template <int TYPE, int N>
__device__ __forceinline__ void load_channels(const Values &v, bool pieces, long row, int column, int end, float (&x)[8 * N]) {
    typedef typename Element<TYPE>::type E;
    if (pieces) {
#pragma unroll
        for (int p = 0; p < N; ++p) {
            union {
                int4 word[sizeof(E) / 2];
                E e[8];
            } u;
#pragma unroll
            for (int k = 0; k < (int)sizeof(E) / 2; ++k) u.word[k] = int4{0, 0, 0, 0};
            if (column + 8 * p < end) {
                const int4 *from = (const int4 *)((const E *)v.data + row * v.stride + column + 8 * p);
#pragma unroll
                for (int k = 0; k < (int)sizeof(E) / 2; ++k) u.word[k] = from[k];
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) x[8 * p + k] = to_float<TYPE>(u.e[k], v.unit, v.p);
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8 * N; ++k) x[k] = column + k < end ? load_value<TYPE>(v, row, column + k) : 0.0f;
    }
}
__device__ __forceinline__ void store_any(const Values &v, long row, int column, float x) {
    switch (v.type) {
        case GALA_F32: store_value<GALA_F32>(v, row, column, x); break;
        case GALA_F16: store_value<GALA_F16>(v, row, column, x); break;
        case GALA_BF16: store_value<GALA_BF16>(v, row, column, x); break;
        default: store_value<GALA_RESIDUE>(v, row, column, x); break;
    }
}

// ND words -> ND planes of balanced base-256 digits of four numbers: the numbers come with 128 added to each digit but
// the highest, as the low bytes of their words
template <int ND>
__device__ __forceinline__ void planes(const u32 (&w)[4], int at, v4i (&to)[ND]) {
    const u32 ab = __builtin_amdgcn_perm(w[1], w[0], 0x05010400), cd = __builtin_amdgcn_perm(w[3], w[2], 0x05010400);
    const u32 low = __builtin_amdgcn_perm(cd, ab, 0x05040100) ^ 0x80808080u, mid = __builtin_amdgcn_perm(cd, ab, 0x07060302);
    to[0][at] = (int)low;
    if constexpr (ND == 2) {
        to[1][at] = (int)mid;
    } else {
        to[1][at] = (int)(mid ^ 0x80808080u);
        const u32 ab2 = __builtin_amdgcn_perm(w[1], w[0], 0x07030602), cd2 = __builtin_amdgcn_perm(w[3], w[2], 0x07030602);
        const u32 third = __builtin_amdgcn_perm(cd2, ab2, 0x05040100);
        if constexpr (ND == 3) {
            to[2][at] = (int)third;
        } else {
            to[2][at] = (int)(third ^ 0x80808080u);
            to[3][at] = (int)__builtin_amdgcn_perm(cd2, ab2, 0x07060302);
        }
    }
}
template <int ND>
struct Digits;
// the largest number, and 128 in every digit but the highest
template <>
struct Digits<2> { static constexpr float most = 127 * 256.0f; static constexpr u32 offset = 128; };
template <>
struct Digits<3> { static constexpr float most = 127 * 65536.0f; static constexpr u32 offset = 128 * 257; };
template <>
struct Digits<4> { static constexpr float most = 127 * 16777216.0f; static constexpr u32 offset = 128 * 65793; };

// the number whose digits' products were added up apart
template <int ND>
__device__ __forceinline__ float joined(const v4i (&acc)[ND], int r) {
    const int low = acc[0][r] + (acc[1][r] << 8);
    if constexpr (ND == 2)
        return (float)low;
    else if constexpr (ND == 3)
        return fmaf((float)acc[2][r], 65536.0f, (float)low);
    else
        return fmaf((float)(acc[2][r] + (acc[3][r] << 8)), 65536.0f, (float)low);
}

// A lane's part of a query, 16 channels of each 64, as digits; returns what a unit of them is worth in exponents of 2,
// with the scale.  `bad`: the query holds a NaN or an infinity; its digits are 0 then.  Two digits round each channel by 2^-16
// of the row's largest, at most a sixteenth of what f16 itself may round that largest by, and less of bf16; three by 2^-24.
template <int NC, int ND>
__device__ __forceinline__ float digits_of(const float (&x)[NC][16], float scale, v4i (&qd)[NC][ND], bool &bad) {
    float most = 0;
    bool fine = true;
#pragma unroll
    for (int k = 0; k < NC; ++k)
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            most = fmaxf(most, fabsf(x[k][j]));
            fine &= fabsf(x[k][j]) < INFINITY;
        }
    most = fmaxf(most, __shfl_xor(most, 16));
    most = fmaxf(most, __shfl_xor(most, 32));
    int all = fine;
    all &= __shfl_xor(all, 16);
    all &= __shfl_xor(all, 32);
    bad = !all;
    const bool some = most > 0 && !bad;
    // a power of two first: the reciprocal of a tiny number would be infinite
    const int e = some ? min(max(ilogbf(most), -126), 126) : 0;
    const float down = ldexpf(1.0f, -e), scaled = some ? most * down : 1.0f, mul = Digits<ND>::most / scaled * (scale < 0 ? -1.0f : 1.0f);
    const float unit_q = ldexpf(scaled / Digits<ND>::most, e) * fabsf(scale) * kLog2E;
#pragma unroll
    for (int k = 0; k < NC; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            u32 w[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int v = some ? (int)rintf(x[k][4 * j + r] * down * mul) : 0;
                w[r] = (u32)v + Digits<ND>::offset;
            }
            planes<ND>(w, j, qd[k]);
        }
    return unit_q;
}

// Both products run on the matrix cores as exact sums of 8-bit products: the cache's codes as they lie in memory by
// the base-256 digits of the queries and of the weights (NC x 64 channels; ND and NW digits).  Of a block's scores a lane has
// 16 of one column's, and they are the very weights that it hands to the second product, because the values' codes
// lie in that order of tokens.  So a block goes from memory to the sums without LDS or an exchange between lanes, but
// for the largest score.  A wavefront has blocks of its own; a workgroup's wavefronts are joined at the end.
// A weight has four digits, 31 bits of the largest in its block: with the two that a query of 16 bits has, thousands of keys that share
// what one heavy key leaves were rounded away (a quarter of the output where the first token has 0.9 of 8192 keys' weight).
// One query a sequence is bound by HBM: 64 sequences of 8192 tokens (8 heads of 128 channels, 807 MB) take 157 us, 5.1 TB/s, the
// matrix cores busy for 0.1 of it; 151 us with two digits.  128 queries of 32 heads over 30000 tokens take 162 us, 124 with two digits.
template <int N32, int ND, int kWaves>
__global__ __launch_bounds__(64 * kWaves, N32 * ND <= 12 ? 2 : 1) void kv_attention_kernel(Attention a) {
    constexpr int NC = (N32 + 1) / 2, NV = 2 * N32;          // products of 64 channels, tiles of 16
    constexpr int NW = 4;                                    // digits of a weight
    __shared__ float sums[kWaves][kColumns][NV * 16 + 1];
    __shared__ float stats[kWaves][kColumns][2];
    const KvArgs &kv = a.kv;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, part = lane >> 4;
    int unit = blockIdx.x;
    const int split = unit % a.splits;
    unit /= a.splits;
    const int tile = unit % a.tiles;
    unit /= a.tiles;
    const int h = unit % kv.heads, b = unit / kv.heads;
    const Seen s = seen_by(a, b, tile);
    if (!s.cols) return;
    const int share = share_of(a, s.total), from = split * share, to = min(s.total, from + share);
    if (split && from >= s.total) return;
    // The next block's keys and scales are under way while this one's weights are made, the one after's page too.
    const size_t head_bytes = kv_head_bytes(kv.dim16);
    v4i keys[4][NC];
    float scale_k = 0, scale_v = 0;
    int u = from + wave, page, page_next;
    auto page_at = [&](int v) { return v < to ? page_of(kv, b, s.block(v)) : -1; };
    auto load_keys = [&]() __attribute__((always_inline)) {
        // without a page the first one is read and not seen: no branch around what is under way
        const size_t head = (size_t)max(page, 0) * kv.heads + h;
        const signed char *codes = kv.codes + head * head_bytes;
        scale_k = kv.scales[2 * head], scale_v = page < 0 ? 0.0f : kv.scales[2 * head + 1];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int k = 0; k < NC; ++k)       // channels beyond the head's meet digits of 0; what is read there is the head's
                keys[i][k] = *(const v4i *)(codes + (size_t)(i * kv.dim16 + k * 4 + part) * 256 + col * 16);
    };
    page = page_at(u), page_next = page_at(u + kWaves);
    if (u < to) load_keys();
    // from block u to the next one
    auto step = [&]() __attribute__((always_inline)) {
        page = page_next;
        load_keys();
        page_next = page_at(u + 2 * kWaves);
    };
    // the column's query: digits, and what one unit of them is worth
    const int c = s.col0 + min(col, s.cols - 1), qi = c / a.group, g = c % a.group;
    const long row = s.start + qi;
    const int at = s.at_lo - s.col0 / a.group + qi, hq = h * a.group + g;
    v4i qd[NC][ND];
    float unit_q;
    bool bad;
    {
        float x[NC][16];
        auto load = [&](auto type) __attribute__((always_inline)) {
#pragma unroll
            for (int k = 0; k < NC; ++k) {
                const int d = k * 64 + part * 16;
                load_channels<decltype(type)::value, 2>(a.q, a.pieces, row, hq * kv.dim + d, hq * kv.dim + kv.dim, x[k]);
            }
        };
        by_type(a.q.type, load);
        unit_q = digits_of<NC, ND>(x, a.scale, qd, bad);
    }
    v4f o[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) o[j] = v4f{0, 0, 0, 0};
    float top = -INFINITY, sum = 0;
    for (; u < to; u += kWaves) {
        const int block = s.block(u), end = page < 0 ? 0 : kv.max_len;
        const signed char *codes = kv.codes + ((size_t)max(page, 0) * kv.heads + h) * head_bytes;
        const float unit_s = unit_q * scale_k, scale_of_v = scale_v;
        v4i values[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j)
            values[j] = *(const v4i *)(codes + (size_t)kKvBlock * 16 * kv.dim16 + min(j, kv.dim16 - 1) * 1024 + lane * 16);
        float t[16];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v4i acc[ND];
#pragma unroll
            for (int n = 0; n < ND; ++n) {
                acc[n] = v4i{0, 0, 0, 0};
#pragma unroll
                for (int k = 0; k < NC; ++k) acc[n] = __builtin_amdgcn_mfma_i32_16x16x64_i8(keys[i][k], qd[k][n], acc[n], 0, 0, 0);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) t[4 * i + r] = joined<ND>(acc, r) * unit_s;
        }
        step();
        const int t0 = block * kKvBlock;
        if (t0 + 63 > s.at_lo || t0 + 64 > end || (a.window && t0 <= s.at_hi - a.window)) {
            // keys of the block by their distance from the lane's first one; no branches between them
            const int own = t0 + part * 4, hi = min(at, end - 1) - own;
            const int lo = a.window ? at - a.window + 1 - own : -kKvBlock, sinks = a.window ? a.sinks - own : 0;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int e = i * 16 + r;
                    t[4 * i + r] = (e <= hi) & ((e >= lo) | (e < sinks)) ? t[4 * i + r] : -INFINITY;
                }
        }
        float most = t[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) most = fmaxf(most, t[i]);
        most = fmaxf(most, __shfl_xor(most, 16));
        most = fmaxf(most, __shfl_xor(most, 32));
        if (__any(most > top)) {
            const float now = fmaxf(top, most), was = now > top ? __builtin_amdgcn_exp2f(top - now) : 1.0f;
            top = now;
            sum *= was;
#pragma unroll
            for (int j = 0; j < NV; ++j) o[j] *= was;
        }
        // Weights as shares of the block's own largest, as whole numbers: a token that outweighs all others by far takes bits from
        // its block's other tokens at most, not from all that come later.
        const float base = most == -INFINITY ? 0.0f : most, part_of = most == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(most - top);
        const float unit_v = scale_of_v * part_of * (1.0f / Digits<NW>::most);
        float part_sum = 0;
        v4i w[NW];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            u32 word[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float p = __builtin_amdgcn_exp2f(t[4 * i + r] - base);
                part_sum += p;
                word[r] = (u32)fmaf(p, Digits<NW>::most, 0.5f) + Digits<NW>::offset;
            }
            planes<NW>(word, i, w);
        }
        sum = fmaf(part_sum, part_of, sum);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            v4i acc[NW];
#pragma unroll
            for (int n = 0; n < NW; ++n) acc[n] = __builtin_amdgcn_mfma_i32_16x16x64_i8(values[j], w[n], v4i{0, 0, 0, 0}, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; ++r) o[j][r] = fmaf(joined<NW>(acc, r), unit_v, o[j][r]);
        }
    }
    // the wavefronts' sums in one
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) sums[wave][col][j * 16 + part * 4 + r] = o[j][r];
    if (part == 0) stats[wave][col][0] = bad ? __builtin_nanf("") : top, stats[wave][col][1] = sum;
    __syncthreads();
    const long place = (((long)b * kv.heads + h) * a.tiles + tile) * a.splits + split;
    for (int e = threadIdx.x; e < s.cols * kv.dim; e += 64 * kWaves) {
        const int cc = e / kv.dim, d = e % kv.dim;
        float most = -INFINITY, all = 0, x = 0;
#pragma unroll
        for (int k = 0; k < kWaves; ++k) most = fmaxf(most, stats[k][cc][0]);
        const float base = most == -INFINITY ? 0.0f : most;
#pragma unroll
        for (int k = 0; k < kWaves; ++k) {
            const float f = __builtin_amdgcn_exp2f(stats[k][cc][0] - base);       // NaN where the query is
            all += f * stats[k][cc][1];
            x += f * sums[k][cc][d];
        }
        if (a.splits == 1) {
            const int column = s.col0 + cc;
            store_any(a.out, s.start + column / a.group, (h * a.group + column % a.group) * kv.dim + d, all == 0 ? 0.0f : x / all);
        } else {
            a.sums[(place * a.columns + cc) * kv.dim + d] = x;
            if (d == 0) a.stats[(place * a.columns + cc) * 2] = all != all ? __builtin_nanf("") : most, a.stats[(place * a.columns + cc) * 2 + 1] = all;
        }
    }
}

// The shares of one query's keys in one: a wavefront takes every eighth share, a lane channels 64 apart.
constexpr int kJoinWaves = 8;
template <int NC>
__global__ __launch_bounds__(64 * kJoinWaves) void kv_attention_join_kernel(Attention a) {
    __shared__ float parts[kJoinWaves][NC * 64 + 1];
    const KvArgs &kv = a.kv;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int unit = blockIdx.x;
    const int cc = unit % a.columns;
    unit /= a.columns;
    const int tile = unit % a.tiles;
    unit /= a.tiles;
    const int h = unit % kv.heads, b = unit / kv.heads;
    const Seen s = seen_by(a, b, tile);
    if (cc >= s.cols) return;
    const int share = share_of(a, s.total), used = share ? max(1, (s.total + share - 1) / share) : 1;
    const long place = (((long)b * kv.heads + h) * a.tiles + tile) * a.splits;
    const float *stats = a.stats + (place * a.columns + cc) * 2, *sums = a.sums + (place * a.columns + cc) * kv.dim;
    const long next = a.columns;
    float most = -INFINITY, all = 0, x[NC];
    for (int k = lane; k < used; k += 64) most = fmaxf(most, stats[k * next * 2]);
    for (int k = 32; k; k >>= 1) most = fmaxf(most, __shfl_xor(most, k));
    const float base = most == -INFINITY ? 0.0f : most;
#pragma unroll
    for (int j = 0; j < NC; ++j) x[j] = 0;
#pragma unroll 4
    for (int k = wave; k < used; k += kJoinWaves) {
        const float f = __builtin_amdgcn_exp2f(stats[k * next * 2] - base);           // NaN where the query is
        all += f * stats[k * next * 2 + 1];
#pragma unroll
        for (int j = 0; j < NC; ++j) x[j] += f * sums[k * next * kv.dim + min(lane + 64 * j, kv.dim - 1)];
    }
#pragma unroll
    for (int j = 0; j < NC; ++j) parts[wave][lane + 64 * j] = x[j];
    if (lane == 0) parts[wave][NC * 64] = all;
    __syncthreads();
    for (int d = threadIdx.x; d < kv.dim; d += 64 * kJoinWaves) {
        float sum = 0, out = 0;
#pragma unroll
        for (int k = 0; k < kJoinWaves; ++k) sum += parts[k][NC * 64], out += parts[k][d];
        const int column = s.col0 + cc;
        store_any(a.out, s.start + column / a.group, (h * a.group + column % a.group) * kv.dim + d, sum == 0 ? 0.0f : out / sum);
    }
}

// ---- many queries of a sequence ---------------------------------------------------------------------------------------
// Here the products and the weights count, not the cache's bytes.  Scores are the same exact sums as above; of the values a
// workgroup makes half-precision fragments in LDS once for its eight wavefronts of a column tile each (the codes are whole
// numbers that half precision holds exactly), so that the second product adds up in 32-bit floats and needs no work
// between blocks.  Its other operand, a weight, is rounded to 11 bits and carries its block's scale of values:
// w = 2^(t + log2(scale) - base), base within 2^8 of the largest so far.  Keys stay 8-bit in LDS: half the reads of
// half-precision fragments.  Wavefronts in their products go before those that make weights.  4096 queries over themselves, 32
// heads of 128 channels: 173 us, 0.79 P a second; bound by the vector ALU, 170 instructions and 16 exponentials for 16 x 64
// scores, which eight wavefronts between two barriers overlap only in part with the products.
// The largest weight is raised to 2^7 and may grow to 2^15, near the end of half precision: so it has 11 bits for weights
// down to 2^-21 of the largest, and steps of 2^-31 of it below.
constexpr int kGroup = 8;
constexpr float kRaised = 7, kHighest = 15;      // exponents
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));

// 16 codes -> 16 half-precision numbers: 1024 + 128 + code is a bit pattern, 1152 is taken off
__device__ __forceinline__ void halves_of(const v4i &codes, v8h (&to)[2]) {
    union {
        u32 word[8];
        v2h pair[8];
        v8h out[2];
    } u;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const u32 w = (u32)codes[k] ^ 0x80808080u;
        u.word[2 * k] = __builtin_amdgcn_perm(0x64646464u, w, 0x04010400);
        u.word[2 * k + 1] = __builtin_amdgcn_perm(0x64646464u, w, 0x04030402);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) u.pair[k] -= v2h{1152, 1152};
    to[0] = u.out[0], to[1] = u.out[1];
}

template <int NK>
__global__ __launch_bounds__(64 * kGroup, NK <= 4 ? 4 : 2) void kv_attention_many_kernel(Attention a) {
    constexpr int NC = (NK + 1) / 2, NV = 2 * NK;    // products of 64 channels of keys, tiles of 16 channels of values
    constexpr int kKeys = NC * 4096, kBuffer = kKeys + NK * 4096;   // keys as they are, values in half precision
    constexpr int kLoads = (2 * NK + kGroup - 1) / kGroup;          // pieces of 16 codes a thread loads, of keys and of values
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const KvArgs &kv = a.kv;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, part = lane >> 4, tid = threadIdx.x;
    // The last queries see most keys: they go first, of all heads (4096 tokens alone 173 us; head after head 223).  A head's groups
    // go to one XCD where there are eight heads.
    int unit = blockIdx.x;
    const int per_group = kv.count * kv.heads, group = a.tiles - 1 - unit / per_group;
    unit %= per_group;
    const int h = unit % kv.heads, b = unit / kv.heads;
    constexpr int kColumnsOf = kGroup * kColumns;
    const Seen s = seen_by(a, b, group, kColumnsOf);
    if (!s.cols) return;
    // the wavefront's queries
    const int c0 = s.col0 + wave * kColumns, c1 = min(c0 + kColumns, s.col0 + s.cols) - 1;
    const int base_at = s.at_lo - s.col0 / a.group, at_lo = base_at + min(c0, c1) / a.group, at_hi = base_at + c1 / a.group;
    const bool idle = c0 > c1;
    int at;
    v4i qd[NC][2];
    float unit_q;
    bool bad;
    {
        const int c = min(c0 + col, s.col0 + s.cols - 1), qi = c / a.group, hq = h * a.group + c % a.group;
        const long row = s.start + qi;
        at = base_at + qi;
        float x[NC][16];
        auto load = [&](auto type) __attribute__((always_inline)) {
#pragma unroll
            for (int k = 0; k < NC; ++k) {
                const int d = k * 64 + part * 16;
                load_channels<decltype(type)::value, 2>(a.q, a.pieces, row, hq * kv.dim + d, hq * kv.dim + kv.dim, x[k]);
            }
        };
        by_type(a.q.type, load);
        unit_q = digits_of<NC, 2>(x, a.scale, qd, bad);
    }
    v4f o[NV];
    float base = 0, limit = -INFINITY, sum = 0;      // limit: what an exponent may be before the base is raised
#pragma unroll
    for (int j = 0; j < NV; ++j) o[j] = v4f{0, 0, 0, 0};
    // channels that fill up a product of 32 are zero in both buffers from here on
    if (kv.dim16 & 1)
        for (int i = tid; i < 2 * 128; i += 64 * kGroup) {
            *(v4i *)(lds + (i >> 7) * kBuffer + kKeys + ((i >> 6 & 1) * NV + NV - 1) * 1024 + (i & 63) * 16) = v4i{0, 0, 0, 0};
        }
    // a block's pieces on their way from the cache to LDS
    const size_t head_bytes = kv_head_bytes(kv.dim16);
    const int pieces = kv.dim16 * 64;
    v4i staged[2][kLoads];
    int key_at[kLoads];          // piece (16 tokens, 16 channels, token)
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
        const int i = tid + k * 64 * kGroup, t16 = (i >> 4) / kv.dim16, d16 = (i >> 4) - t16 * kv.dim16;
        key_at[k] = (t16 * 4 * NC + d16) * 256 + (i & 15) * 16;
    }
    float scale_k = 0, scale_v = 0;
    int page = -1, page_next = 0;
    // the page of block u has to be there when its codes are asked for: it is asked for a block earlier
    auto page_at = [&](int u) __attribute__((always_inline)) { return u < s.total ? page_of(kv, b, s.block(u)) : -1; };
    auto fetch = [&](int u) __attribute__((always_inline)) {
        page = __builtin_amdgcn_readfirstlane(page_next);
        const size_t head = (size_t)max(page, 0) * kv.heads + h;
        const signed char *codes = kv.codes + head * head_bytes;
        const float2 scales = *(const float2 *)(kv.scales + 2 * head);
        scale_k = scales.x, scale_v = scales.y;
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            const int i = min(tid + k * 64 * kGroup, pieces - 1);
            staged[0][k] = ((const v4i *)codes)[i];
            staged[1][k] = ((const v4i *)codes)[pieces + i];
        }
        page_next = page_at(u + 1);
    };
    page_next = page_at(0);
    if (s.total) fetch(0);
    for (int u = 0; u < s.total; ++u) {
        char *keys = lds + (u & 1) * kBuffer, *values = keys + kKeys;
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            if (tid + k * 64 * kGroup < pieces) {
                *(v4i *)(keys + key_at[k]) = staged[0][k];
                // values: the first and the last 32 tokens of a channel
                v8h x[2];
                halves_of(staged[1][k], x);
                char *to = values + (tid + k * 64 * kGroup) * 16;
                *(v8h *)to = x[0], *(v8h *)(to + NV * 1024) = x[1];
            }
        }
        const int block = s.block(u), t0 = block * kKvBlock, end = page < 0 ? 0 : kv.max_len;
        // Values of nothing get a scale that is small, but does not take their weights, which count in the sum, out of 32 bits.
        const float now_k = scale_k, now_v = page < 0 ? 1.0f : scale_v >= 0x1p-100f ? scale_v : 0x1p-64f;
        if (u + 1 < s.total) fetch(u + 1);
        __syncthreads();
        if (idle || t0 > at_hi || t0 >= end || (a.window && t0 + 63 <= at_lo - a.window && t0 >= a.sinks)) continue;
        const bool edge = t0 + 63 > at_lo || t0 + 64 > end || (a.window && t0 <= at_hi - a.window);
        const float log_v = __builtin_amdgcn_logf(now_v), unit_l = __builtin_amdgcn_exp2f(-kRaised) / now_v;
        __builtin_amdgcn_s_setprio(1);
        v4f acc[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v4i sums[2];
#pragma unroll
            for (int n = 0; n < 2; ++n) sums[n] = v4i{0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < NC; ++k) {       // channels beyond the head's meet digits of 0
                const v4i x = *(const v4i *)(keys + (i * NC + k) * 1024 + lane * 16);
#pragma unroll
                for (int n = 0; n < 2; ++n) sums[n] = __builtin_amdgcn_mfma_i32_16x16x64_i8(x, qd[k][n], sums[n], 0, 0, 0);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[i][r] = joined<2>(sums, r);
        }
        __builtin_amdgcn_s_setprio(0);
        v8h w[2];
        const float unit_s = fmaxf(unit_q * now_k, 0x1p-126f);      // not 0: what is not seen stays at -infinity
        if (edge) {
            const int own = t0 + part * 4, hi = min(at, end - 1) - own;
            const int lo = a.window ? at - a.window + 1 - own : -kKvBlock, sinks = a.window ? a.sinks - own : 0;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int e = i * 16 + r;
                    acc[i][r] = (e <= hi) & ((e >= lo) | (e < sinks)) ? acc[i][r] : -INFINITY;
                }
        }
        // exponents below the base so far
        const float off = log_v - base;
        float most = -INFINITY;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                acc[i][r] = fmaf(acc[i][r], unit_s, off);
                most = fmaxf(most, acc[i][r]);
            }
        if (__any(most > limit)) {
            most = fmaxf(most, __shfl_xor(most, 16));
            most = fmaxf(most, __shfl_xor(most, 32));
            if (most > limit || most > kRaised) {
                most -= kRaised;
                const float was = limit == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(-most);          // nothing yet with the first base
                base += most;
                limit = kHighest;
                sum *= was;
#pragma unroll
                for (int j = 0; j < NV; ++j) o[j] *= was;
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[i] -= most;
            }
        }
        // the values' fragments four ahead of the products
        auto fragment = [&](int f) __attribute__((always_inline)) { return *(const v8h *)(values + ((f & 1) * NV + (f >> 1)) * 1024 + lane * 16); };
        v8h ahead[4];
#pragma unroll
        for (int f = 0; f < 4; ++f) ahead[f] = fragment(f);
        float part_sum = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float x = __builtin_amdgcn_exp2f(acc[i][r]);
                part_sum += x;
                w[i >> 1][(i & 1) * 4 + r] = (_Float16)x;
            }
        sum = fmaf(part_sum, unit_l, sum);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int f = 0; f < 2 * NV; ++f) {
            o[f >> 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ahead[f & 3], w[f & 1], o[f >> 1], 0, 0, 0);
            if (f + 4 < 2 * NV) ahead[f & 3] = fragment(f + 4);
        }
        __builtin_amdgcn_s_setprio(0);
    }
    float all = sum;
    all += __shfl_xor(all, 16);
    all += __shfl_xor(all, 32);
    const float f = bad ? __builtin_nanf("") : all > 0 ? 1.0f / all : 0.0f;
    // the sum is that of weights with a largest of 1: its reciprocal stays a normal number
    auto lowered = [](float x) __attribute__((always_inline)) { return x * __builtin_amdgcn_exp2f(-kRaised); };
    const int c = c0 + col;
    if (c > c1) return;
    const long row = s.start + c / a.group;
    const int column = (h * a.group + c % a.group) * kv.dim + part * 4;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int d = j * 16 + part * 4;
        if (d + 4 <= kv.dim && a.out_quads) {
            auto store = [&](auto type) __attribute__((always_inline)) {
                typedef typename Element<decltype(type)::value>::type E;
                struct alignas(4 * sizeof(E) < 16 ? 4 * sizeof(E) : 16) Quad {
                    E e[4];
                } quad;
#pragma unroll
                for (int r = 0; r < 4; ++r) quad.e[r] = from_float<decltype(type)::value>(lowered(o[j][r]) * f, a.out.unit, a.out.p);
                *(Quad *)((E *)a.out.data + row * a.out.stride + column + j * 16) = quad;
            };
            by_type(a.out.type, store);
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (d + r < kv.dim) store_any(a.out, row, column + j * 16 + r, lowered(o[j][r]) * f);
        }
    }
}

// How a call is cut up.
struct Cut {
    bool many;
    int tiles, splits, columns;
    long places() const { return (long)tiles * splits * columns; }
};
Cut cut_of(const KvArgs &kv, int heads_q, int window, int sinks, bool fine) {
    Cut c;
    const int group = heads_q / kv.heads;
    const long columns = (long)kv.max_new * group;
    const int of_group = kGroup * kColumns;
    const long reach = std::min<long>(kv.max_len, (long)kv.table_stride * kKvBlock);
    const long keys = window ? std::min(reach, (long)window + kv.max_new + sinks + 2 * kKvBlock) : reach;
    const long blocks = std::max(1l, (keys + kKvBlock - 1) / kKvBlock);
    // The call's bound on new tokens decides for all of its sequences, and a token beside a prompt then shares its keys with nobody:
    // a prompt of 2000 and 15 single tokens over 8192 tokens take 1029 us, in two calls 325.  Whole prompts in half precision,
    // where they fill the card or have few keys: 8 x 128 queries of 32 heads over 4000 tokens (256 workgroups) take 105 us so and
    // 179 us as exact sums, 4 x 300 over 300 14 and 33 us; but 4 x 128 over 4000 (128 workgroups) 104 and 91 us, because exact
    // sums can share a tile's keys.
    const long groups = (columns + of_group - 1) / of_group * kv.count * kv.heads;
    c.many = !fine && columns >= of_group && (groups >= 192 || blocks <= 16);
    if (c.many) {
        c.tiles = (int)((columns + of_group - 1) / of_group), c.splits = 1, c.columns = 0;
        return c;
    }
    c.tiles = (int)((columns + kColumns - 1) / kColumns);
    c.columns = (int)std::min<long>(columns, kColumns);
    // Workgroups for one round of the card, with 32 blocks at least: 64 sequences of 8192 tokens take 157 us in 512 workgroups,
    // 173 us in 1024 and 177 us in 4096.
    const long units = std::max(1l, (long)kv.count * kv.heads * c.tiles);
    c.splits = (int)std::max(1l, std::min((512 + units - 1) / units, (blocks + 31) / 32));
    return c;
}

}  // namespace

namespace gala {

size_t kv_attention_workspace(const KvArgs &kv, int heads_q, int window, int sinks) {
    const Cut c = cut_of(kv, heads_q, window, sinks, true);          // the other way needs none
    return c.splits == 1 ? 0 : (size_t)kv.count * kv.heads * c.places() * (kv.dim + 2) * sizeof(float);
}

int launch_kv_attention(void *stream, const KvArgs &kv, int heads_q, float scale, int window, int sinks, const Values &q,
                        const Values &out, void *workspace) {
    const bool fine = q.type == GALA_F32 || q.type == GALA_RESIDUE || out.type == GALA_F32 || out.type == GALA_RESIDUE;
    const Cut c = cut_of(kv, heads_q, window, sinks, fine);
    Attention a{};
    a.kv = kv, a.q = q, a.out = out;
    const size_t size = q.type == GALA_F32 ? 4 : q.type == GALA_RESIDUE ? 8 : 2;
    a.pieces = (uintptr_t)q.data % 16 == 0 && q.stride * size % 16 == 0 && kv.dim % 8 == 0;
    const size_t of_out = out.type == GALA_F32 ? 4 : out.type == GALA_RESIDUE ? 8 : 2, quad = std::min<size_t>(4 * of_out, 16);
    a.out_quads = (uintptr_t)out.data % quad == 0 && out.stride * of_out % quad == 0 && kv.dim % 4 == 0;
    a.heads_q = heads_q, a.group = heads_q / kv.heads;
    a.scale = scale, a.window = window, a.sinks = sinks;
    a.tiles = c.tiles, a.splits = c.splits, a.columns = c.columns;
    a.sums = (float *)workspace;
    a.stats = a.sums + (size_t)kv.count * kv.heads * c.places() * kv.dim;
    const unsigned groups = (unsigned)((long)kv.count * kv.heads * c.tiles * c.splits);
    auto launch = [&](auto n32) {
        constexpr int N32 = decltype(n32)::value, NC = (N32 + 1) / 2;
        if (c.many) {
            hipLaunchKernelGGL((kv_attention_many_kernel<N32>), dim3(groups), dim3(64 * kGroup), 2 * (NC + N32) * 4096, (hipStream_t)stream, a);
            return;
        }
        // A launch that leaves CUs with one workgroup gets eight wavefronts in each: 32 windows of 1024 tokens take 12.4 us with
        // eight and 15.0 with four; 64 sequences of 500 tokens in 512 workgroups 18.1 and 14.5.
        auto waves = [&](auto w) {
            constexpr int W = decltype(w)::value;
            a.waves = W;
            if (fine)
                hipLaunchKernelGGL((kv_attention_kernel<N32, 3, W>), dim3(groups), dim3(64 * W), 0, (hipStream_t)stream, a);
            else
                hipLaunchKernelGGL((kv_attention_kernel<N32, 2, W>), dim3(groups), dim3(64 * W), 0, (hipStream_t)stream, a);
        };
        if constexpr (N32 <= 4) {
            if (groups <= 256)
                waves(std::integral_constant<int, 8>());
            else
                waves(std::integral_constant<int, 4>());
        } else {
            waves(std::integral_constant<int, 4>());
        }
        if (c.splits == 1) return;
        const unsigned rows = (unsigned)((long)kv.count * kv.heads * c.tiles * c.columns);
        hipLaunchKernelGGL(kv_attention_join_kernel<NC>, dim3(rows), dim3(64 * kJoinWaves), 0, (hipStream_t)stream, a);
    };
    switch ((kv.dim + 31) / 32) {
        case 1: launch(std::integral_constant<int, 1>()); break;
        case 2: launch(std::integral_constant<int, 2>()); break;
        case 3: launch(std::integral_constant<int, 3>()); break;
        case 4: launch(std::integral_constant<int, 4>()); break;
        case 5: launch(std::integral_constant<int, 5>()); break;
        case 6: launch(std::integral_constant<int, 6>()); break;
        case 7: launch(std::integral_constant<int, 7>()); break;
        default: launch(std::integral_constant<int, 8>()); break;
    }
    return hipGetLastError() != hipSuccess;
}

}  // namespace gala
