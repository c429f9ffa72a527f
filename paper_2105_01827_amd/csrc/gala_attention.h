// Attention over a paged cache: what its kernels for codes of 8 and of 4 bits have in common.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "gala_decode.h"

namespace gala {
namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));

struct Attention {
    KvArgs kv;
    Values q, out;
    bool pieces, out_quads;          // rows of q lie on 16 bytes, those of out on four values
    int heads_q, group;              // group: query heads of a head of the cache
    float scale;
    int window, sinks;
    int waves;                       // wavefronts of a workgroup
    bool ordered;                    // groups of queries of all sequences go by what they see
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

}  // namespace
}  // namespace gala
