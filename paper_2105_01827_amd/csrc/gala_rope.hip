// Rotary positions with several axes into rows of heads: the pair (u, v) of channels becomes (c u - s v, c v + s u) with the cosine and
// sine of its axis' position.  A read and a write of the rows: bound by HBM (9801 rows of 32 heads of 80 f16 channels, 100 MB, 26 us: 3.8 TB/s; 6000
// of 32 of 128 in bfloat16, 98 MB, 22.2 us: 4.4), by the launch where rows are few (8 rows 4.2 us).
#include "gala_rows.h"

using namespace gala;

namespace {

constexpr int kThreads = 256;

struct Axes {
    gala_rope_axes rope;
    const int *at;
    long at_stride;
    int rows, heads, dim;
};

// A row's place on its axes; none where the table lacks one of them.
struct Place {
    int at[4];
    bool has;
};
__device__ __forceinline__ Place place_of(const Axes &a, long row) {
    Place p;
    p.has = true;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        p.at[k] = k < a.rope.axes ? a.at[row * a.at_stride + k] : 0;
        p.has &= (u32)p.at[k] < (u32)a.rope.positions;
    }
    return p;
}
// `pair`: its axis, and 4 times its column
__device__ __forceinline__ float2 angle_of(const Axes &a, const Place &p, u32 pair) {
    const int axis = pair & 3, at = axis == 0 ? p.at[0] : axis == 1 ? p.at[1] : axis == 2 ? p.at[2] : p.at[3];
    return *(const float2 *)(a.rope.table + ((long)at * a.rope.columns + (pair >> 2)) * 2);
}
template <int TYPE, int OUT>
__global__ __launch_bounds__(kThreads) void rope_apply_kernel(Axes a, Turns turns, Values x, Values out) {
    __shared__ u32 pairs[128];
    const int half = a.rope.rot_dim / 2;
    if ((int)threadIdx.x < half) pairs[threadIdx.x] = a.rope.axis[threadIdx.x] | (u32)a.rope.column[threadIdx.x] << 2;
    __syncthreads();
    const long first = (long)(blockIdx.x / turns.parts) * turns.rows;
    turn_heads<TYPE, OUT, kThreads>(turns, blockIdx.x % turns.parts, x, out, [&](int r) { return first + r < a.rows ? first + r : -1; },
                                    [&](int r, bool two, bool turned, int d, float(&angle)[16]) __attribute__((always_inline)) {
        const Place p = place_of(a, first + r);
        if (p.has && turned) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k < 4 || two) {
                    const float2 x = angle_of(a, p, pairs[two ? d + k : d / 2 + k]);
                    angle[2 * k] = x.x, angle[2 * k + 1] = x.y;
                }
        }
        return p.has;
    });
}
// The same for rows of any size and place, a number at a load: a row a workgroup, a pair or a number behind them a thread.
template <int TYPE, int OUT>
__global__ __launch_bounds__(kThreads) void rope_apply_any_kernel(Axes a, Values x, Values out) {
    __shared__ u32 pairs[128];
    const int half = a.rope.rot_dim / 2, rest = a.dim - half;
    if ((int)threadIdx.x < half) pairs[threadIdx.x] = a.rope.axis[threadIdx.x] | (u32)a.rope.column[threadIdx.x] << 2;
    __syncthreads();
    const long row = blockIdx.x;
    const Place p = place_of(a, row);
    for (int e = threadIdx.x; e < a.heads * rest; e += kThreads) {
        const int h = e / rest, k = e - h * rest;
        if (k < half) {
            const int d = a.rope.interleaved ? 2 * k : k, other = a.rope.interleaved ? d + 1 : d + half;
            float u = load_value<TYPE>(x, row, h * a.dim + d), v = load_value<TYPE>(x, row, h * a.dim + other);
            if (p.has) {
                const float2 x = angle_of(a, p, pairs[k]);
                turn_pair(x.x, x.y, u, v);
            }
            store_value<OUT>(out, row, h * a.dim + d, p.has ? u : __builtin_nanf(""));
            store_value<OUT>(out, row, h * a.dim + other, p.has ? v : __builtin_nanf(""));
        } else {
            const float u = load_value<TYPE>(x, row, h * a.dim + half + k);
            store_value<OUT>(out, row, h * a.dim + half + k, p.has ? u : __builtin_nanf(""));
        }
    }
}

}  // namespace

namespace gala {

int launch_rope_apply(void *stream, const gala_rope_axes &rope, const int *at, long at_stride, int rows, int heads, int dim, const Values &x,
                      const Values &out) {
    const bool whole = in_pieces(x, dim) && in_pieces(out, dim) && rope.rot_dim / 2 % (rope.interleaved ? 4 : 8) == 0;
    const Axes a{rope, at, at_stride, rows, heads, dim};
    const Turns turns = turns_of(rows, heads, dim, rope.rot_dim / 2, rope.interleaved, kThreads);
    by_type(x.type, [&](auto type) {
        by_type(out.type, [&](auto o) {
            constexpr int T = decltype(type)::value, O = decltype(o)::value;
            if constexpr (O != GALA_RESIDUE) {
                if (whole)
                    hipLaunchKernelGGL((rope_apply_kernel<T, O>), dim3((rows + turns.rows - 1) / turns.rows * turns.parts), dim3(kThreads), 0, (hipStream_t)stream, a,
                                       turns, x, out);
                else
                    hipLaunchKernelGGL((rope_apply_any_kernel<T, O>), dim3(rows), dim3(kThreads), 0, (hipStream_t)stream, a, x, out);
            }
        });
    });
    return hipGetLastError() != hipSuccess;
}

}  // namespace gala
