// One token a row from logits and given uniform numbers.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "gala_decode.h"

using namespace gala;

namespace {

constexpr int kThreads = 1024;
constexpr float kWeightOne = 1099511627776.0f;      // 2^40

// A logit's place in descending order: the larger, the smaller; both zeros alike.
__device__ __forceinline__ u32 descending(float z) {
    const u32 bits = __float_as_uint(z + 0.0f);
    return ~((bits & 0x80000000u) ? ~bits : bits | 0x80000000u);
}

struct Shared {
    u64 bins[256];
    u64 carry, total;
    u32 digit;
    float part[16];
};

// Of elements with keys and weights, given by each(f(key, weight)) over all threads together, the key at which the
// weights added up in ascending order of keys first exceed `target`: digit by digit from the top, in sums of the
// weights of all elements whose digits so far are the key's.  Needs target < the sum of all.
template <class E>
__device__ u64 weighted_select(Shared &sh, u64 target, int bits, E each) {
    u64 prefix = 0;
    for (int shift = (bits + 7) / 8 * 8 - 8; shift >= 0; shift -= 8) {
        for (int i = threadIdx.x; i < 256; i += kThreads) sh.bins[i] = 0;
        __syncthreads();
        each([&](u64 key, u64 weight) {
            if (weight && (shift + 8 >= 64 || key >> (shift + 8) == prefix >> (shift + 8)))
                atomicAdd((unsigned long long *)&sh.bins[key >> shift & 255], (unsigned long long)weight);
        });
        __syncthreads();
        if (threadIdx.x == 0) {
            u64 before = 0;
            int digit = 0;
            while (digit < 255 && before + sh.bins[digit] <= target) before += sh.bins[digit++];
            sh.digit = digit, sh.carry = before;
        }
        __syncthreads();
        prefix |= (u64)sh.digit << shift;
        target -= sh.carry;
        __syncthreads();
    }
    return prefix;
}

// One workgroup a row.
template <int TYPE>
__global__ __launch_bounds__(kThreads) void sample_kernel(Values logits, int vocab, gala_sampling how, int *tokens) {
#pragma clang fp contract(off)
    __shared__ Shared sh;
    const int row = blockIdx.x, tid = threadIdx.x;
    auto logit = [&](int i) { return load_value<TYPE>(logits, row, i); };
    const float temperature = how.temperature ? how.temperature[row] : 1.0f;
    const bool greedy = temperature <= 0;
    const float rate = greedy ? 1.0f : 1.0f / temperature;
    float top = -INFINITY;
    for (int i = tid; i < vocab; i += kThreads) top = fmaxf(top, logit(i));        // a NaN is never the larger
    for (int k = 32; k; k >>= 1) top = fmaxf(top, __shfl_xor(top, k));
    if ((tid & 63) == 0) sh.part[tid >> 6] = top;
    __syncthreads();
    for (int k = 0; k < kThreads / 64; ++k) top = fmaxf(top, sh.part[k]);
    if (top == -INFINITY) {
        if (tid == 0) tokens[row] = -1;
        return;
    }
    auto chance = [&](float z) { return z == top ? 1.0f : z == z ? expf((z - top) * rate) : 0.0f; };
    auto weight = [&](float z) { return (u64)(chance(z) * kWeightOne); };
    auto key = [&](float z, int i) { return (u64)descending(z) << 32 | (u32)i; };
    auto sum_of = [&](auto f) {
        if (tid == 0) sh.total = 0;
        __syncthreads();
        u64 sum = 0;
        for (int i = tid; i < vocab; i += kThreads) sum += f(logit(i), i);
        for (int k = 32; k; k >>= 1) sum += __shfl_xor(sum, k);
        if ((tid & 63) == 0) atomicAdd((unsigned long long *)&sh.total, (unsigned long long)sum);
        __syncthreads();
        const u64 all = sh.total;
        __syncthreads();
        return all;
    };
    u64 last = ~0ull;                                                             // the last key that is kept
    const int most = greedy ? 1 : how.top_k ? how.top_k[row] : 0;
    if (most > 0 && most < vocab) {
        auto each = [&](auto f) {
            for (int i = tid; i < vocab; i += kThreads) {
                const float z = logit(i);
                f(key(z == z ? z : -INFINITY, i), (u64)1);
            }
        };
        last = weighted_select(sh, most - 1, 64, each);
    }
    const float share = how.top_p ? how.top_p[row] : 1.0f, given = how.min_p ? how.min_p[row] : 0.0f;
    const float least = given == given ? fminf(given, 1.0f) : 0.0f;
    if (share < 1) {
        const u64 all = sum_of([&](float z, int i) { return key(z, i) <= last ? weight(z) : (u64)0; });
        const double below = ceil((double)share * (double)all) - 1;
        auto each = [&](auto f) {
            for (int i = tid; i < vocab; i += kThreads) {
                const float z = logit(i);
                if (key(z, i) <= last) f(key(z, i), weight(z));
            }
        };
        last = weighted_select(sh, below > 0 ? min((u64)below, all - 1) : 0, 64, each);
    }
    auto kept = [&](float z, int i) {
        const float w = chance(z);
        return key(z, i) <= last && w >= least ? (u64)(w * kWeightOne) : (u64)0;
    };
    const u64 all = sum_of(kept);
    const double drawn = (double)how.u[row] * (double)all;
    const u64 target = drawn > 0 ? min((u64)drawn, all - 1) : 0;
    auto each = [&](auto f) {
        for (int i = tid; i < vocab; i += kThreads) f((u64)i, kept(logit(i), i));
    };
    const int bits = 32 - __clz(vocab);
    const u64 token = weighted_select(sh, target, bits, each);
    if (tid == 0) tokens[row] = (int)token;
}

}  // namespace

namespace gala {

size_t sample_workspace(int, int) { return 0; }

int launch_sample(void *stream, const Values &logits, int rows, int vocab, const gala_sampling &how, int *tokens, void *) {
    by_type(logits.type, [&](auto type) {
        hipLaunchKernelGGL(sample_kernel<decltype(type)::value>, dim3(rows), dim3(kThreads), 0, (hipStream_t)stream, logits, vocab, how,
                           tokens);
    });
    return hipGetLastError() != hipSuccess;
}

}  // namespace gala
