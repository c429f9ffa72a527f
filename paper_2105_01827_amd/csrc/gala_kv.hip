// Keys and values of new tokens into the paged 8-bit cache, positions rotated in on the way, and rows of the cache
// back as floats.
#include <hip/hip_runtime.h>

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

// Bound by HBM in prompts and by the launch for single tokens.  A workgroup has a whole block of a head, so that the
// scale it needs is found and used in one launch and the rows are read once.
template <int TYPE, int OUT>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(KvArgs kv, RopeArgs rope, int heads_q, Values q, Values q_out, Values k,
                                                             Values v, int blocks, int units) {
    __shared__ float tile[kKvBlock][kChunk + 1];
    __shared__ float shared[4];
    const int unit = blockIdx.x;
    if (unit < units)
        append_block<TYPE>(kv, rope, unit & 1 ? v : k, unit, blocks, tile, shared);
    else
        rotate_row<TYPE, OUT>(kv, rope, q, q_out, heads_q, unit - units);
}

// One workgroup: the keys or the values of one head in one block of one sequence.
template <int OUT>
__global__ __launch_bounds__(kThreads) void kv_export_kernel(KvArgs kv, Values k_out, Values v_out, int blocks) {
    const int unit = blockIdx.x;
    const int which = unit & 1, h = (unit >> 1) % kv.heads, bj = (unit >> 1) / kv.heads, b = bj / blocks, j = bj % blocks;
    const int start = kv.starts[b], n = kv.starts[b + 1] - start, first = kv.lens[b] - n;
    // tokens at negative positions are in blocks of their own numbers, down from -1
    const int block = (first >= 0 ? first / kKvBlock : -((63 - first) / kKvBlock)) + j, at = block * kKvBlock;
    const int lo = max(first, at), hi = min(first + min(n, kv.max_new), at + kKvBlock);
    if (lo >= hi) return;
    const int page = page_of(kv, b, block);
    const Values &out = which ? v_out : k_out;
    const float scale = page < 0 ? 0.0f : kv.scales[((long)page * kv.heads + h) * 2 + which];
    const signed char *codes = page < 0 ? nullptr : kv.codes + ((long)page * kv.heads + h) * kv_head_bytes(kv.dim16) + (which ? kKvBlock * 16 * kv.dim16 : 0);
    for (int e = threadIdx.x; e < (hi - lo) * kv.dim; e += kThreads) {
        const int t = lo - at + e / kv.dim, d = e % kv.dim;
        const int place = which ? (d >> 4) * 1024 + ((t & 15) >> 2) * 256 + (d & 15) * 16 + (t >> 4) * 4 + (t & 3)
                                : ((t >> 4) * kv.dim16 + (d >> 4)) * 256 + (t & 15) * 16 + (d & 15);
        const float x = page < 0 ? 0.0f : (float)codes[place] * scale;
        store_value<OUT>(out, start + (at + t - first), h * kv.dim + d, x);
    }
}

}  // namespace

namespace gala {

int launch_kv_append(void *stream, const KvArgs &kv, const RopeArgs &rope, int heads_q, const Values &q, const Values &q_out,
                     const Values &k, const Values &v) {
    // the most blocks that max_new tokens in a row can touch
    const int blocks = (kv.max_new + kKvBlock - 2) / kKvBlock + 1, units = k.data ? kv.count * blocks * kv.heads * 2 : 0;
    const int rows = heads_q ? kv.count * kv.max_new : 0;
    by_type(k.data ? k.type : q.type, [&](auto type) {
        by_type(q_out.type, [&](auto out) {
            constexpr int T = decltype(type)::value, O = decltype(out)::value;
            if constexpr (O != GALA_RESIDUE)
                hipLaunchKernelGGL((kv_append_kernel<T, O>), dim3(units + rows), dim3(kThreads), 0, (hipStream_t)stream, kv, rope,
                                   heads_q, q, q_out, k, v, blocks, units);
        });
    });
    return hipGetLastError() != hipSuccess;
}

int launch_kv_export(void *stream, const KvArgs &kv, const Values &k_out, const Values &v_out) {
    const int blocks = (kv.max_new + kKvBlock - 2) / kKvBlock + 1;
    by_type(k_out.type, [&](auto type) {
        hipLaunchKernelGGL(kv_export_kernel<decltype(type)::value>, dim3(kv.count * blocks * kv.heads * 2), dim3(kThreads), 0,
                           (hipStream_t)stream, kv, k_out, v_out, blocks);
    });
    return hipGetLastError() != hipSuccess;
}

}  // namespace gala
