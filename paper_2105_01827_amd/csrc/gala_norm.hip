// A layer's output added to the residual stream, and the root-mean-square norm of the sum in few bits for the next layer.
#include <cmath>

#include "gala_rows.h"

using namespace gala;

namespace {

// value k of a thread, and eight of them at a time
template <bool PIECES, int THREADS>
__device__ __forceinline__ int column_of(int tid, int k) {
    return PIECES ? (k / 8 * THREADS + tid) * 8 + k % 8 : k * THREADS + tid;
}
// N x 8 numbers of a row as floats, 0 behind its end
template <bool PIECES, int THREADS, int N>
__device__ __forceinline__ void load_row(const Values &v, long row, int tid, int width, float (&x)[8 * N]) {
    by_type(v.type, [&](auto type) __attribute__((always_inline)) {
        constexpr int T = decltype(type)::value;
        typedef typename Element<T>::type E;
        if constexpr (PIECES) {
            union Piece {
                int4 word[sizeof(E) / 2];
                E e[8];
            } u[N];
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const int column = column_of<true, THREADS>(tid, 8 * n);
                const int4 *from = (const int4 *)((const E *)v.data + row * v.stride + (column < width ? column : 0));
#pragma unroll
                for (int k = 0; k < (int)sizeof(E) / 2; ++k) u[n].word[k] = from[k];
            }
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int k = 0; k < 8; ++k) x[8 * n + k] = column_of<true, THREADS>(tid, 8 * n) < width ? to_float<T>(u[n].e[k], v.unit, v.p) : 0.0f;
        } else {
            E e[8 * N];
#pragma unroll
            for (int k = 0; k < 8 * N; ++k) {
                const int column = column_of<false, THREADS>(tid, k);
                e[k] = ((const E *)v.data)[row * v.stride + (column < width ? column : 0)];
            }
#pragma unroll
            for (int k = 0; k < 8 * N; ++k) x[k] = column_of<false, THREADS>(tid, k) < width ? to_float<T>(e[k], v.unit, v.p) : 0.0f;
        }
    });
}
template <bool PIECES, int THREADS, int N>
__device__ __forceinline__ void store_row(const Values &v, long row, int tid, int width, const float (&x)[8 * N]) {
    by_type(v.type, [&](auto type) __attribute__((always_inline)) {
        constexpr int T = decltype(type)::value;
        if constexpr (PIECES) {
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const int column = column_of<true, THREADS>(tid, 8 * n);
                float piece[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) piece[k] = x[8 * n + k];
                if (column < width) store_piece<T>(v, row, column, piece);
            }
        } else {
#pragma unroll
            for (int k = 0; k < 8 * N; ++k) {
                const int column = column_of<false, THREADS>(tid, k);
                if (column < width) store_value<T>(v, row, column, x[k]);
            }
        }
    });
}
// whole numbers, as int8 or as residues
template <bool PIECES, int THREADS, int N>
__device__ __forceinline__ void store_codes(const Values &v, long row, int tid, int width, const float (&x)[8 * N]) {
    auto residue = [&](float c) { return (u64)((long)c + (c < 0 ? (long)v.p : 0)); };
#pragma unroll
    for (int k = 0; k < 8 * N; k += PIECES ? 8 : 1) {
        const int column = column_of<PIECES, THREADS>(tid, k);
        if (column >= width) continue;
        if (v.type == GALA_INT8) {
            signed char *to = (signed char *)v.data + row * v.stride + column;
            if constexpr (PIECES) {
                u32 w[2] = {0, 0};
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i / 4] |= (u32)((int)x[k + i] & 255) << 8 * (i % 4);
                *(uint2 *)to = uint2{w[0], w[1]};
            } else {
                *to = (signed char)(int)x[k];
            }
        } else {
            u64 *to = (u64 *)v.data + row * v.stride + column;
#pragma unroll
            for (int i = 0; i < (PIECES ? 8 : 1); i += PIECES ? 2 : 1) {
                if constexpr (PIECES)
                    *(ulong2 *)(to + i) = ulong2{residue(x[k + i]), residue(x[k + i + 1])};
                else
                    *to = residue(x[k]);
            }
        }
    }
}

__device__ __forceinline__ float code_of(float y, float inverse, float limit) {
    const float t = rintf(y * inverse);
    return t != t ? 0.0f : fminf(limit, fmaxf(-limit, t));
}

struct Rows {
    NormArgs how;
    Values x, add, sum, weight, out;
};

// A row stays in the registers of THREADS threads, N pieces of eight numbers each: one pass over memory.  Rows of up to a wavefront's
// registers share a workgroup of four.
template <int THREADS, int N, bool PIECES>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void rms_norm_kernel(Rows a) {
#pragma clang fp contract(off)
    constexpr int kWaves = THREADS / 64, kRows = THREADS < 256 ? 256 / THREADS : 1;
    static_assert(THREADS == 64 || THREADS >= 256, "a wavefront or a workgroup");
    extern __shared__ u32 largest[];             // of every group of every row
    __shared__ double sums[kWaves];
    const NormArgs &how = a.how;
    const int tid = threadIdx.x % THREADS, width = how.width;
    const long row = (long)blockIdx.x * kRows + threadIdx.x / THREADS;
    const bool idle = kRows > 1 && row >= how.rows;
    const int groups = how.scales ? (width + how.group - 1) / how.group : 0;
    u32 *slots = largest + (threadIdx.x / THREADS) * groups;
    for (int g = tid; g < groups; g += THREADS) slots[g] = 0;
    if constexpr (kWaves == 1) __syncthreads();          // else the sum's
    float s[8 * N], other[8 * N];
    if (!idle) {
        load_row<PIECES, THREADS, N>(a.x, row, tid, width, s);
        if (a.add.data) {
            load_row<PIECES, THREADS, N>(a.add, row, tid, width, other);
#pragma unroll
            for (int k = 0; k < 8 * N; ++k) s[k] += other[k];
        }
        if (a.weight.data) {
            load_row<PIECES, THREADS, N>(a.weight, 0, tid, width, other);
        } else {
#pragma unroll
            for (int k = 0; k < 8 * N; ++k) other[k] = 1;
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8 * N; ++k) s[k] = other[k] = 0;
    }
    double all = 0;
#pragma unroll
    for (int k = 0; k < 8 * N; ++k) all = fma((double)s[k], (double)s[k], all);
    for (int k = 32; k; k >>= 1) all += __shfl_xor(all, k);
    if constexpr (kWaves > 1) {
        if ((tid & 63) == 0) sums[tid >> 6] = all;
        __syncthreads();
        all = 0;
#pragma unroll
        for (int k = 0; k < kWaves; ++k) all += sums[k];
    }
    if (!idle && a.sum.data) store_row<PIECES, THREADS, N>(a.sum, row, tid, width, s);
    const float factor = (float)(1.0 / sqrt(all / width + how.epsilon));
#pragma unroll
    for (int k = 0; k < 8 * N; ++k) s[k] = s[k] * factor * other[k];
    if (a.out.type < GALA_RESIDUE) {
        if (!idle) store_row<PIECES, THREADS, N>(a.out, row, tid, width, s);
        return;
    }
    if (!how.scales) {
#pragma unroll
        for (int k = 0; k < 8 * N; ++k) {
            const float t = rintf(s[k] / a.out.unit);
            s[k] = t != t ? 0.0f : fminf(how.limit, fmaxf(-how.limit, t));
        }
        if (!idle) store_codes<PIECES, THREADS, N>(a.out, row, tid, width, s);
        return;
    }
    // the largest magnitude of every group
    auto finite = [](float y) { return fabsf(y) < INFINITY ? fabsf(y) : 0.0f; };
    if (groups == 1) {
        float most = 0;
#pragma unroll
        for (int k = 0; k < 8 * N; ++k) most = fmaxf(most, finite(s[k]));
        for (int k = 32; k; k >>= 1) most = fmaxf(most, __shfl_xor(most, k));
        if ((tid & 63) == 0) atomicMax(&slots[0], __float_as_uint(most));
    } else {
#pragma unroll
        for (int k = 0; k < 8 * N; k += PIECES ? 8 : 1) {
            const int column = column_of<PIECES, THREADS>(tid, k);
            float most = finite(s[k]);
#pragma unroll
            for (int i = 1; i < (PIECES ? 8 : 1); ++i) most = fmaxf(most, finite(s[k + i]));
            if (column < width) atomicMax(&slots[column / how.group], __float_as_uint(most));
        }
    }
    __syncthreads();
    if (idle) return;
    for (int g = tid; g < groups; g += THREADS) how.scales[row * groups + g] = __uint_as_float(slots[g]) * how.step;
#pragma unroll
    for (int k = 0; k < 8 * N; k += PIECES ? 8 : 1) {
        const int column = column_of<PIECES, THREADS>(tid, k);
        const float scale = column < width ? __uint_as_float(slots[column / how.group]) * how.step : 0.0f;
        const float inverse = scale > 0 ? 1.0f / scale : 0.0f;
#pragma unroll
        for (int i = 0; i < (PIECES ? 8 : 1); ++i) s[k + i] = code_of(s[k + i], inverse, how.limit);
    }
    store_codes<PIECES, THREADS, N>(a.out, row, tid, width, s);
}

// Rows that no workgroup's registers hold, or whose groups are too many for LDS: the row is read three times, nothing is written
// before the last.
__global__ __launch_bounds__(1024) void rms_norm_long_kernel(Rows a) {
#pragma clang fp contract(off)
    __shared__ double sums[16];
    __shared__ u32 largest[16];
    const NormArgs &how = a.how;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, width = how.width;
    const long row = blockIdx.x;
    auto value = [&](const Values &v, long row, int column) {
        float x = 0;
        by_type(v.type, [&](auto type) { x = load_value<decltype(type)::value>(v, row, column); });
        return x;
    };
    auto sum_at = [&](int c) { return a.add.data ? value(a.x, row, c) + value(a.add, row, c) : value(a.x, row, c); };
    double all = 0;
    for (int c = tid; c < width; c += 1024) {
        const double s = sum_at(c);
        all = fma(s, s, all);
    }
    for (int k = 32; k; k >>= 1) all += __shfl_xor(all, k);
    if (lane == 0) sums[wave] = all;
    __syncthreads();
    all = 0;
    for (int k = 0; k < 16; ++k) all += sums[k];
    const float factor = (float)(1.0 / sqrt(all / width + how.epsilon));
    auto normed = [&](float s, int c) { return s * factor * (a.weight.data ? value(a.weight, 0, c) : 1.0f); };
    auto put = [&](int c, float s, float y, float inverse) {
        if (a.sum.data) by_type(a.sum.type, [&](auto type) { store_value<decltype(type)::value>(a.sum, row, c, s); });
        if (a.out.type < GALA_RESIDUE) {
            by_type(a.out.type, [&](auto type) { store_value<decltype(type)::value>(a.out, row, c, y); });
            return;
        }
        float t = how.scales ? rintf(y * inverse) : rintf(y / a.out.unit);
        t = t != t ? 0.0f : fminf(how.limit, fmaxf(-how.limit, t));
        if (a.out.type == GALA_INT8)
            ((signed char *)a.out.data)[row * a.out.stride + c] = (signed char)(int)t;
        else
            ((u64 *)a.out.data)[row * a.out.stride + c] = (u64)((long)t + (t < 0 ? (long)a.out.p : 0));
    };
    if (!how.scales) {
        for (int c = tid; c < width; c += 1024) {
            const float s = sum_at(c);
            put(c, s, normed(s, c), 0);
        }
        return;
    }
    // one group: all wavefronts together; several: each wavefront takes groups of its own
    const int groups = (width + how.group - 1) / how.group;
    const bool together = groups == 1;
    for (int g = together ? 0 : wave; g < groups; g += together ? 1 : 16) {
        const long lo = (long)g * how.group;
        const int hi = (int)min((long)width, lo + how.group), step = together ? 1024 : 64;
        float most = 0;
        for (int c = (int)lo + (together ? tid : lane); c < hi; c += step) {
            const float y = fabsf(normed(sum_at(c), c));
            if (y < INFINITY) most = fmaxf(most, y);
        }
        for (int k = 32; k; k >>= 1) most = fmaxf(most, __shfl_xor(most, k));
        if (together) {
            if (lane == 0) largest[wave] = __float_as_uint(most);
            __syncthreads();
            for (int k = 0; k < 16; ++k) most = fmaxf(most, __uint_as_float(largest[k]));
        }
        const float scale = most * how.step, inverse = scale > 0 ? 1.0f / scale : 0.0f;
        if (together ? tid == 0 : lane == 0) how.scales[row * groups + g] = scale;
        for (int c = (int)lo + (together ? tid : lane); c < hi; c += step) {
            const float s = sum_at(c);
            put(c, s, normed(s, c), inverse);
        }
    }
}

}  // namespace

namespace gala {

int launch_rms_norm(void *stream, const NormArgs &how, const Values &x, const Values &add, const Values &sum, const Values &weight,
                    const Values &out) {
    const int width = how.width;
    Rows a{how, x, add, sum, weight, out};
    hipStream_t st = (hipStream_t)stream;
    const bool int8 = out.type == GALA_INT8;
    const bool pieces = in_pieces(x, width) && in_pieces(add, width) && in_pieces(sum, width) && in_pieces(weight, width) &&
                        (int8 ? (uintptr_t)out.data % 8 == 0 && out.stride % 8 == 0 : in_pieces(out, width)) && (!how.scales || how.group % 8 == 0 || how.group >= width);
    const int groups = how.scales ? (width + how.group - 1) / how.group : 0;
    if (width > 16384 || groups > 8192) {
        hipLaunchKernelGGL(rms_norm_long_kernel, dim3(how.rows), dim3(1024), 0, st, a);
        return hipGetLastError() != hipSuccess;
    }
    auto launch = [&](auto threads, auto n) {
        constexpr int T = decltype(threads)::value, N = decltype(n)::value, R = T < 256 ? 256 / T : 1;
        const dim3 grid((how.rows + R - 1) / R), block(T * R);
        if (pieces)
            hipLaunchKernelGGL((rms_norm_kernel<T, N, true>), grid, block, R * groups * 4, st, a);
        else
            hipLaunchKernelGGL((rms_norm_kernel<T, N, false>), grid, block, R * groups * 4, st, a);
    };
    const std::integral_constant<int, 1> one;
    const std::integral_constant<int, 2> two;
    if (width <= 512)
        launch(std::integral_constant<int, 64>(), one);
    else if (width <= 2048)
        launch(std::integral_constant<int, 256>(), one);
    else if (width <= 4096)
        launch(std::integral_constant<int, 256>(), two);
    else if (width <= 8192)
        launch(std::integral_constant<int, 512>(), two);
    else
        launch(std::integral_constant<int, 1024>(), two);
    return hipGetLastError() != hipSuccess;
}

}  // namespace gala
