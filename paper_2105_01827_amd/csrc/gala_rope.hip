// Rotary positions with several axes into rows of heads.
#include "gala_rows.h"

using namespace gala;

namespace {

constexpr int kThreads = 256;

struct Axes {
    gala_rope_axes rope;
    const int *at;
    long at_stride;
    int rows, heads, dim;
    int slots, rows_of;          // threads that share a row's heads for each piece, rows of a workgroup
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
// products and sums rounded one by one
__device__ __forceinline__ void turn_pair(float2 angle, float &x, float &y) {
#pragma clang fp contract(off)
    const float a = angle.x * x - angle.y * y, b = angle.x * y + angle.y * x;
    x = a, y = b;
}

// A thread takes a piece of a row, in the half layout both members of eight pairs, finds its angles once and turns it in
// every `slots`-th head.
template <int TYPE, int OUT>
__global__ __launch_bounds__(kThreads) void rope_apply_kernel(Axes a, Values x, Values out, Pieces pieces) {
    __shared__ u32 pairs[128];
    const int half = a.rope.rot_dim / 2;
    if ((int)threadIdx.x < half) pairs[threadIdx.x] = a.rope.axis[threadIdx.x] | (u32)a.rope.column[threadIdx.x] << 2;
    __syncthreads();
    const int each = pieces.pairs + pieces.singles, in_row = each * a.slots;
    const Divisor of_row(in_row), of_each(each);
    for (int e = threadIdx.x; e < a.rows_of * in_row; e += kThreads) {
        const int r = of_row(e), rest = e - r * in_row, slot = of_each(rest), piece = rest - slot * each;
        const long row = (long)blockIdx.x * a.rows_of + r;
        if (row >= a.rows) break;
        const Place p = place_of(a, row);
        const bool two = piece < pieces.pairs;
        const int d = two ? piece * 8 : (pieces.pairs + piece) * 8;          // singles lie behind both members of the pairs
        const bool turned = p.has && d < a.rope.rot_dim;
        float2 angle[8];
        if (turned) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k < 4 || two) angle[k] = angle_of(a, p, pairs[two ? d + k : d / 2 + k]);
        }
#pragma unroll 2
        for (int h = slot; h < a.heads; h += a.slots) {
            float u[8], v[8];
            load_piece<TYPE>(x, row, h * a.dim + d, u);
            if (two) load_piece<TYPE>(x, row, h * a.dim + half + d, v);
            if (turned) {
                if (two) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) turn_pair(angle[k], u[k], v[k]);
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k) turn_pair(angle[k], u[2 * k], u[2 * k + 1]);
                }
            }
            if (!p.has) {
#pragma unroll
                for (int k = 0; k < 8; ++k) u[k] = v[k] = __builtin_nanf("");
            }
            store_piece<OUT>(out, row, h * a.dim + d, u);
            if (two) store_piece<OUT>(out, row, h * a.dim + half + d, v);
        }
    }
}
// The same for rows of any size and place: a row a workgroup, a pair or a number behind them a thread.
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
            if (p.has) turn_pair(angle_of(a, p, pairs[k]), u, v);
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
    const Pieces pieces(dim, rope.rot_dim / 2, rope.interleaved);
    const int each = pieces.pairs + pieces.singles;
    const bool whole = in_pieces(x, dim) && in_pieces(out, dim) && rope.rot_dim / 2 % (rope.interleaved ? 4 : 8) == 0;
    Axes a{rope, at, at_stride, rows, heads, dim, 0, 0};
    if (whole) {
        const long turns = std::min(2l, std::max(1l, (long)rows * each * heads / (256 * 512)));        // heads of a thread
        a.slots = (int)((heads + turns - 1) / turns);
        a.slots = std::min(a.slots, std::max(1, 32768 / each));
        a.rows_of = std::max(1, kThreads / (each * a.slots));
    }
    by_type(x.type, [&](auto type) {
        by_type(out.type, [&](auto o) {
            constexpr int T = decltype(type)::value, O = decltype(o)::value;
            if constexpr (O != GALA_RESIDUE) {
                if (whole)
                    hipLaunchKernelGGL((rope_apply_kernel<T, O>), dim3((rows + a.rows_of - 1) / a.rows_of), dim3(kThreads), 0, (hipStream_t)stream, a, x, out,
                                       pieces);
                else
                    hipLaunchKernelGGL((rope_apply_any_kernel<T, O>), dim3(rows), dim3(kThreads), 0, (hipStream_t)stream, a, x, out);
            }
        });
    });
    return hipGetLastError() != hipSuccess;
}

}  // namespace gala
