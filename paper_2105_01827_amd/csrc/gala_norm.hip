// A layer's output added to the residual stream, and the root-mean-square norm of the sum in few bits for the next layer.
#include <cmath>

#include "gala_rows.h"

using namespace gala;

namespace {

// Threads take pieces of eight numbers of a row.  WHOLE: rows lie on 16 bytes and end with a piece.  Else a piece is read where it
// lies -- the loads take any address -- and the numbers of a last one that is not whole one by one.
template <int THREADS>
__device__ __forceinline__ int column_of(int tid, int n) { return (n * THREADS + tid) * 8; }
template <bool WHOLE>
struct alignas(WHOLE ? 16 : 1) Word16 {
    u64 x, y;
} __attribute__((packed));

// N pieces on their way, as they lie in memory
template <int N>
struct Raw {
    u64 word[N][16];
};
template <bool WHOLE, int THREADS, int N>
__device__ __forceinline__ void fetch_row(const Values &v, long row, int tid, int width, Raw<N> &raw) {
    by_type(v.type, [&](auto type) __attribute__((always_inline)) {
        typedef typename Element<decltype(type)::value>::type E;
        const E *from = (const E *)v.data + row * v.stride;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int column = column_of<THREADS>(tid, n);
            if (WHOLE || column + 8 <= width) {
                const Word16<WHOLE> *at = (const Word16<WHOLE> *)(from + (WHOLE && column >= width ? 0 : column));
#pragma unroll
                for (int k = 0; k < (int)sizeof(E) / 2; ++k) {
                    const Word16<WHOLE> w = at[k];
                    raw.word[n][2 * k] = w.x, raw.word[n][2 * k + 1] = w.y;
                }
            } else {
                union {
                    u64 word[sizeof(E)];
                    E e[8];
                } u;
#pragma unroll
                for (int k = 0; k < 8; ++k) u.e[k] = from[min(column + k, width - 1)];
#pragma unroll
                for (int k = 0; k < (int)sizeof(E); ++k) raw.word[n][k] = u.word[k];
            }
        }
    });
}
// ... and as floats, 0 behind the row's end
template <int THREADS, int N>
__device__ __forceinline__ void floats_of(const Values &v, int tid, int width, const Raw<N> &raw, float (&x)[8 * N]) {
    by_type(v.type, [&](auto type) __attribute__((always_inline)) {
        constexpr int T = decltype(type)::value;
        typedef typename Element<T>::type E;
        constexpr int kIn = 8 / sizeof(E);           // numbers of a word
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                E e;
                const u64 word = raw.word[n][k / kIn] >> (k % kIn * 8 * sizeof(E));
                __builtin_memcpy(&e, &word, sizeof(E));
                x[8 * n + k] = column_of<THREADS>(tid, n) + k < width ? to_float<T>(e, v.unit, v.p) : 0.0f;
            }
    });
}
// eight numbers of a row to their places
template <bool WHOLE, class E>
__device__ __forceinline__ void store_eight(E *to, int column, int width, const E (&e)[8]) {
    if (WHOLE ? column < width : column + 8 <= width) {
        if constexpr (sizeof(E) == 1) {
            struct alignas(WHOLE ? 8 : 1) Word8 {
                u64 x;
            } __attribute__((packed)) w;
            __builtin_memcpy(&w, e, 8);
            *(Word8 *)(to + column) = w;
        } else {
#pragma unroll
            for (int k = 0; k < (int)sizeof(E) / 2; ++k) {
                Word16<WHOLE> w;
                __builtin_memcpy(&w, e + k * (16 / sizeof(E)), 16);
                ((Word16<WHOLE> *)(to + column))[k] = w;
            }
        }
    } else if (!WHOLE) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (column + k < width) to[column + k] = e[k];
    }
}
template <bool WHOLE, int THREADS, int N>
__device__ __forceinline__ void store_row(const Values &v, long row, int tid, int width, const float (&x)[8 * N]) {
    by_type(v.type, [&](auto type) __attribute__((always_inline)) {
        constexpr int T = decltype(type)::value;
        typedef typename Element<T>::type E;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            E e[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) e[k] = from_float<T>(x[8 * n + k], v.unit, v.p);
            store_eight<WHOLE>((E *)v.data + row * v.stride, column_of<THREADS>(tid, n), width, e);
        }
    });
}
// whole numbers, as int8 or as residues
template <bool WHOLE, int THREADS, int N>
__device__ __forceinline__ void store_codes(const Values &v, long row, int tid, int width, const float (&x)[8 * N]) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const int column = column_of<THREADS>(tid, n);
        if (v.type == GALA_INT8) {
            signed char e[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) e[k] = (signed char)(int)x[8 * n + k];
            store_eight<WHOLE>((signed char *)v.data + row * v.stride, column, width, e);
        } else {
            u64 e[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int c = (int)x[8 * n + k];
                e[k] = (u64)(c < 0 ? c + (int)v.p : c);
            }
            store_eight<WHOLE>((u64 *)v.data + row * v.stride, column, width, e);
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

// A row stays in the registers of THREADS threads, N pieces of eight numbers each: one pass over memory, which bounds long calls (8191 rows
// of 4096 bf16 numbers, 236 MB, 50 us: 4.7 TB/s; rows off 16 bytes 77 us, their stores split lines).  Few rows are a launch and one chain
// of loads, a sum over the workgroup and stores (1 x 2048 4.2 us, 64 x 5120 5.1 us).  Rows of up to a wavefront's registers share
// a workgroup of four.  The sum of squares is kept in 64 bits: its rounding to the 32-bit factor then is the same in any order of
// addition but for one case in 2^28 or so, and codes with it.
template <int THREADS, int N, bool WHOLE>
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
    const long from = idle ? how.rows - 1 : row;
    {
        // all of the row, and the weights, on their way together: rows of 8191 x 4096 in 52 us, one after the other in 63
        Raw<N> raw, raw_add, raw_weight;
        fetch_row<WHOLE, THREADS, N>(a.x, from, tid, width, raw);
        if (a.add.data) fetch_row<WHOLE, THREADS, N>(a.add, from, tid, width, raw_add);
        if (a.weight.data) fetch_row<WHOLE, THREADS, N>(a.weight, 0, tid, width, raw_weight);
        floats_of<THREADS, N>(a.x, tid, width, raw, s);
        if (a.add.data) {
            floats_of<THREADS, N>(a.add, tid, width, raw_add, other);
#pragma unroll
            for (int k = 0; k < 8 * N; ++k) s[k] += other[k];
        }
        if (a.weight.data) floats_of<THREADS, N>(a.weight, tid, width, raw_weight, other);
    }
    if (!a.weight.data) {
#pragma unroll
        for (int k = 0; k < 8 * N; ++k) other[k] = 1;
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
    if (!idle && a.sum.data) store_row<WHOLE, THREADS, N>(a.sum, row, tid, width, s);
    const float factor = (float)rsqrt(all * how.per_width + how.epsilon);
#pragma unroll
    for (int k = 0; k < 8 * N; ++k) s[k] = s[k] * factor * other[k];
    if (a.out.type < GALA_RESIDUE) {
        if (!idle) store_row<WHOLE, THREADS, N>(a.out, row, tid, width, s);
        return;
    }
    if (!how.scales) {
#pragma unroll
        for (int k = 0; k < 8 * N; ++k) {
            const float t = rintf(s[k] / a.out.unit);
            s[k] = t != t ? 0.0f : fminf(how.limit, fmaxf(-how.limit, t));
        }
        if (!idle) store_codes<WHOLE, THREADS, N>(a.out, row, tid, width, s);
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
    } else if (how.group % 8 == 0) {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            float most = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) most = fmaxf(most, finite(s[8 * n + k]));
            const int column = column_of<THREADS>(tid, n);
            if (column < width) atomicMax(&slots[column / how.group], __float_as_uint(most));
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8 * N; ++k) {
            const int column = column_of<THREADS>(tid, k / 8) + k % 8;
            if (column < width) atomicMax(&slots[column / how.group], __float_as_uint(finite(s[k])));
        }
    }
    __syncthreads();
    if (idle) return;
    for (int g = tid; g < groups; g += THREADS) how.scales[row * groups + g] = __uint_as_float(slots[g]) * how.step;
    auto inverse_of = [&](int column) __attribute__((always_inline)) {
        const float scale = column < width ? __uint_as_float(slots[column / how.group]) * how.step : 0.0f;
        return scale > 0 ? 1.0f / scale : 0.0f;
    };
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const int column = column_of<THREADS>(tid, n);
        const bool together = groups == 1 || how.group % 8 == 0;
        float inverse = inverse_of(column);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (k && !together) inverse = inverse_of(column + k);
            s[8 * n + k] = code_of(s[8 * n + k], inverse, how.limit);
        }
    }
    store_codes<WHOLE, THREADS, N>(a.out, row, tid, width, s);
}

// Rows that no workgroup's registers hold, or whose groups are too many for LDS: the row is read three times, a number a
// load, and nothing is written before the last.  1000 rows of 20000 bf16 numbers to codes take 237 us, 252 with a scale for 128, where the bytes
// are 28 us; 64 of 32768 83 us; 1000 of 20000 f32 numbers to f32 153 us.
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
    const float factor = (float)rsqrt(all * how.per_width + how.epsilon);
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
    const bool whole = in_pieces(x, width) && in_pieces(add, width) && in_pieces(sum, width) && in_pieces(weight, width) &&
                       (out.type == GALA_INT8 ? (uintptr_t)out.data % 8 == 0 && out.stride % 8 == 0 && width % 8 == 0 : in_pieces(out, width));
    const int groups = how.scales ? (width + how.group - 1) / how.group : 0;
    if (width > 16384 || groups > 8192) {
        hipLaunchKernelGGL(rms_norm_long_kernel, dim3(how.rows), dim3(1024), 0, st, a);
        return hipGetLastError() != hipSuccess;
    }
    auto launch = [&](auto threads, auto n) {
        constexpr int T = decltype(threads)::value, N = decltype(n)::value, R = T < 256 ? 256 / T : 1;
        const dim3 grid((how.rows + R - 1) / R), block(T * R);
        if (whole)
            hipLaunchKernelGGL((rms_norm_kernel<T, N, true>), grid, block, R * groups * 4, st, a);
        else
            hipLaunchKernelGGL((rms_norm_kernel<T, N, false>), grid, block, R * groups * 4, st, a);
    };
    const std::integral_constant<int, 1> one;
    const std::integral_constant<int, 2> two;
    // One or two pieces a thread, a wavefront a row where one holds it: with four pieces 1000 x 8192 take 20.1 us instead of 17.8, 1000 x 16384 37.8
    // instead of 34.4, 4000 x 2048 20.3 (a wavefront a row) instead of 15.8; with one instead of two 1000 x 8192 22.5, 8191 x 4095
    // 81 instead of 78.5 (64 x 4096 4.6 instead of 5.1).
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
