// One token a row from logits and given uniform numbers.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "gala_decode.h"

using namespace gala;

// A row's tokens are put into bins by how far their logit is below the largest, a cut is found from the bins' counts
// and weights, and only the bin that the cut falls into is looked at token by token.  A row is shared by several
// workgroups, and each step that needs all of them is a launch of its own:
//   best    the largest logit of every workgroup's part of the row;
//   bins    counts and weights of the bins, where the row has a top-k or top-p;
//   gather  of every chunk, the weight of the tokens that are kept for sure, and a list of those in the cut's bin;
//   draw    the cut within its bin, the chunk that the uniform number falls into, and the token in it.
// Weights are whole numbers, at most 2^40 each of less than 2^24, so the sums do not depend on who adds what first.
// Many long rows are bound by HBM (256 of 131072 residues: 268 MB read twice in 105 us of 113), fewer by the vector ALU (64 of
// 100003 with top-p: 44 instructions a logit in `bins`, 12.7 of 36.7 us), one row by its four launches (2.9, 4.6, 6.0
// and 10.0 us for 32000 logits).  A cut among more tokens of a bin than a list holds is searched digit by digit by one workgroup:
// top-p of 0.95 among 131072 logits of a long tail takes 51 us at temperature 1 and 566 us at 1.3.
namespace {

constexpr int kThreads = 512, kDrawThreads = 512;
constexpr float kWeightOne = 1099511627776.0f;      // 2^40
// 1/32 of a factor e each; from the last bin on weights are less than 2^-40 and count as nothing
constexpr int kBins = 896;
constexpr float kBinsPerUnit = 32.0f;
constexpr int kListed = 2048;                       // tokens of a list; a row that needs more is searched as a whole
// Longest list that is put in order by counting: a list of a few tokens takes 23.3 us of one row's time so and 27.0 us through the
// network.
constexpr int kCounted = 128;
constexpr int kMostChunks = 256;

// A logit's place in descending order: the larger, the smaller; both zeros alike.
__device__ __forceinline__ u32 descending(float z) {
    const u32 bits = __float_as_uint(z + 0.0f);
    return ~((bits & 0x80000000u) ? ~bits : bits | 0x80000000u);
}
__device__ __forceinline__ float logit_of(u64 key) {
    const u32 bits = ~(u32)(key >> 32);
    return __uint_as_float((bits & 0x80000000u) ? bits & 0x7fffffffu : ~bits);
}
__device__ __forceinline__ u64 key_of(float z, int i) { return (u64)descending(z == z ? z : -INFINITY) << 32 | (u32)i; }

struct Workspace {
    u64 *mass;               // rows x kBins: weights, and of every bin the count
    u32 *count;
    u32 *listed;             // rows: tokens of the list, those beyond its end included
    u64 *list;               // rows x kListed keys
    u64 *best;               // rows x groups
    u64 *sure;               // rows x chunks
};
struct Sample {
    Values logits;
    int rows, vocab;
    int groups;              // workgroups of a row, each has `each` chunks
    int each, chunks, chunk; // chunk: tokens of a chunk, 1 << shift
    int shift;
    gala_sampling how;
    int *tokens;
    Workspace ws;
    // a chunk's first token: chunks but the first begin on 16 bytes
    template <int TYPE>
    __device__ int from(int row, int c) const {
        typedef typename Element<TYPE>::type E;
        constexpr int kOf = 16 / sizeof(E);
        const int off = (int)((uintptr_t)((const E *)logits.data + row * logits.stride) / sizeof(E) % kOf);
        return c == 0 ? 0 : c >= chunks ? vocab : min(vocab, c * chunk + (off ? kOf - off : 0));
    }
};

// What a row asks for.
struct Row {
    float top, rate, share, least;
    int first;               // the first token, -1 if the row has none
    int most;                // top-k, 0: all
    bool greedy;

    __device__ float chance(float z) const {
#pragma clang fp contract(off)
        return z == top ? 1.0f : z > -INFINITY ? expf((z - top) * rate) : 0.0f;
    }
    __device__ u64 weight(float z) const { return (u64)(chance(z) * kWeightOne); }
    __device__ int bin(float z) const { 
#pragma clang fp contract(off)
        return z == top ? 0 : z == z ? (int)fminf((z - top) * rate * -kBinsPerUnit, kBins - 1) : kBins - 1;
    }
    // 0 where the token is not kept for its weight
    __device__ u64 kept(float z) const {
        const float w = chance(z);
        return w >= least ? (u64)(w * kWeightOne) : (u64)0;
    }
    __device__ bool cuts() const { return !greedy && first >= 0 && (most > 0 || share < 1); }
};
// Reductions over a wavefront's lanes by data-parallel moves: within rows of 16 lanes, then from row to row.  The
// exchange through LDS that shuffles take is ten times the latency, and these kernels are chains of such steps.
template <int CTRL, int ROWS>
__device__ __forceinline__ u64 moved(u64 v, u64 none) {
    const u32 low = __builtin_amdgcn_update_dpp((int)none, (int)v, CTRL, ROWS, 0xf, false);
    const u32 high = __builtin_amdgcn_update_dpp((int)(none >> 32), (int)(v >> 32), CTRL, ROWS, 0xf, false);
    return (u64)high << 32 | low;
}
template <class F>
__device__ __forceinline__ u64 scanned(u64 v, u64 none, F f) {
    v = f(v, moved<0x111, 0xf>(v, none));        // from 1, 2, 4 and 8 lanes below in the row
    v = f(v, moved<0x112, 0xf>(v, none));
    v = f(v, moved<0x114, 0xf>(v, none));
    v = f(v, moved<0x118, 0xf>(v, none));
    v = f(v, moved<0x142, 0xa>(v, none));        // rows 1 and 3 from the last lane of the row below
    v = f(v, moved<0x143, 0xc>(v, none));        // rows 2 and 3 from lane 31
    return v;
}
__device__ __forceinline__ u64 from_lane(u64 v, int lane) {
    return (u64)(u32)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (u32)__builtin_amdgcn_readlane((int)v, lane);
}
// over the wavefront's lanes up to the own one
__device__ __forceinline__ u64 upto_of(u64 v) {
    return scanned(v, 0, [](u64 a, u64 b) { return a + b; });
}
__device__ __forceinline__ u64 wave_sum(u64 v) { return from_lane(upto_of(v), 63); }
__device__ __forceinline__ u64 wave_min(u64 v) {
    return from_lane(scanned(v, ~0ull, [](u64 a, u64 b) { return min(a, b); }), 63);
}
// by every wavefront for itself, from the largest logits of the row's parts
__device__ __forceinline__ Row row_of(const Sample &a, int row) {
    Row r;
    u64 best = ~0ull;
    for (int i = threadIdx.x & 63; i < a.groups; i += 64) best = min(best, a.ws.best[(long)row * a.groups + i]);
    best = wave_min(best);
    const float temperature = a.how.temperature ? a.how.temperature[row] : 1.0f, least = a.how.min_p ? a.how.min_p[row] : 0.0f;
    r.top = logit_of(best);
    r.first = r.top == -INFINITY ? -1 : (int)(u32)best;
    r.greedy = temperature <= 0;
    r.rate = r.greedy ? 1.0f : 1.0f / temperature;
    r.share = a.how.top_p ? a.how.top_p[row] : 1.0f;
    r.least = least == least ? fminf(least, 1.0f) : 0.0f;
    const int most = a.how.top_k ? a.how.top_k[row] : 0;
    r.most = most > 0 && most < a.vocab ? most : 0;
    return r;
}

// The logits of a row from `lo` to `hi`: 16 bytes a load where they lie on 16 bytes, several loads under way together,
// and what is before and behind them one by one.
struct Nothing {
    __device__ void operator()(int, int) const {}
};
template <int TYPE, int THREADS>
struct Logits {
    typedef typename Element<TYPE>::type E;
    static constexpr int kOf = 16 / sizeof(E), kLoads = TYPE == GALA_RESIDUE ? 8 : 4;
    union Vector {
        int4 word;
        E e[kOf];
    };
    const Values &logits;
    const E *x;
    int lo, hi, begin, vectors, behind;

    __device__ __forceinline__ Logits(const Values &logits, int row, int lo, int hi) : logits(logits), lo(lo), hi(hi) {
        x = (const E *)logits.data + row * logits.stride;
        const int off = (int)((uintptr_t)(x + lo) / sizeof(E) % kOf);
        begin = min(hi, lo + (off ? kOf - off : 0)), vectors = (hi - begin) / kOf, behind = begin + vectors * kOf;
    }
    // f(logit, index), a thread's in ascending order.  After each load done(index, next): the first index of the
    // wavefront's 64 loads and of its next ones, neither beyond the last logit; behind the last load next is -1.
    template <class F, class D = Nothing>
    __device__ __forceinline__ void each(F f, D done = D()) {
        const int tid = threadIdx.x;
        auto value = [&](E e) { return to_float<TYPE>(e, logits.unit, logits.p); };
        if (lo + tid < begin) f(value(x[lo + tid]), lo + tid);
        for (int at = tid; at - (tid & 63) < vectors; at += kLoads * THREADS) {
            Vector v[kLoads];
#pragma unroll
            for (int k = 0; k < kLoads; ++k) v[k].word = *(const int4 *)(x + begin + (long)min(at + k * THREADS, vectors - 1) * kOf);
#pragma unroll
            for (int k = 0; k < kLoads; ++k) {
                if (at + k * THREADS < vectors)
#pragma unroll
                    for (int j = 0; j < kOf; ++j) f(value(v[k].e[j]), begin + (at + k * THREADS) * kOf + j);
                const int here = begin + (at - (tid & 63) + k * THREADS) * kOf;
                done(min(here, hi - 1), min(here + THREADS * kOf, hi - 1));
            }
        }
        if (behind + tid < hi) f(value(x[behind + tid]), behind + tid);
        done(hi - 1, -1);
    }
};

template <int TYPE>
__global__ __launch_bounds__(kThreads) void sample_best_kernel(Sample a) {
    __shared__ u64 part[kThreads / 64];
    const int row = blockIdx.x / a.groups, c = blockIdx.x % a.groups, tid = threadIdx.x;
    float top = -INFINITY;
    int first = -1;
    Logits<TYPE, kThreads> logits(a.logits, row, a.from<TYPE>(row, c * a.each), a.from<TYPE>(row, (c + 1) * a.each));
    logits.each([&](float z, int i) {
        if (z > top) top = z, first = i;
    });
    u64 best = wave_min(key_of(top, first));
    if ((tid & 63) == 0) part[tid >> 6] = best;
    // what the next launches add to
    for (int i = c * kThreads + tid; i < kBins; i += a.groups * kThreads) a.ws.mass[(long)row * kBins + i] = 0, a.ws.count[(long)row * kBins + i] = 0;
    if (c == 0 && tid == 0) a.ws.listed[row] = 0;
    __syncthreads();
    if (tid == 0) {
        for (int k = 1; k < kThreads / 64; ++k) best = min(best, part[k]);
        a.ws.best[(long)row * a.groups + c] = best;
    }
}

__device__ __forceinline__ bool asks_to_cut(const Sample &a, int row) {
    const int most = a.how.top_k ? a.how.top_k[row] : 0;
    return (most > 0 && most < a.vocab) || (a.how.top_p && a.how.top_p[row] < 1);
}
template <int TYPE>
__global__ __launch_bounds__(kThreads) void sample_bins_kernel(Sample a) {
    __shared__ u64 mass[kBins];
    __shared__ u32 count[kBins];
    const int row = blockIdx.x / a.groups, c = blockIdx.x % a.groups;
    if (!asks_to_cut(a, row)) return;
    Logits<TYPE, kThreads> logits(a.logits, row, a.from<TYPE>(row, c * a.each), a.from<TYPE>(row, (c + 1) * a.each));
    const Row r = row_of(a, row);
    if (!r.cuts()) return;
    for (int i = threadIdx.x; i < kBins; i += kThreads) mass[i] = 0, count[i] = 0;
    __syncthreads();
    const bool counts = r.most > 0, weighs = r.share < 1;
    logits.each([&](float z, int) {
        const int bin = r.bin(z);
        if (bin == kBins - 1) return;            // what is left over is in the last one
        if (counts) atomicAdd(&count[bin], 1u);
        if (weighs) atomicAdd((unsigned long long *)&mass[bin], (unsigned long long)r.weight(z));
    });
    __syncthreads();
    for (int i = threadIdx.x; i < kBins; i += kThreads) {
        if (count[i]) atomicAdd(&a.ws.count[(long)row * kBins + i], count[i]);
        if (mass[i]) atomicAdd((unsigned long long *)&a.ws.mass[(long)row * kBins + i], (unsigned long long)mass[i]);
    }
}

// The bins up to each, and the cuts as far as the bins tell.
struct Bins {
    u64 mass[kBins];         // of the bin and all before it
    u32 count[kBins];
    u64 part_mass[16];
    u32 part_count[16];
    int k_bin, p_low, p_high;
};
// Tokens of bins below `sure` are kept (min-p apart); those of bins in [low, high] and of k_bin are to be looked at.
struct Cut {
    int sure, low, high, k_bin;
    bool by_k;
    __device__ bool open(int bin) const { return (bin >= low && bin <= high) || (by_k && bin == k_bin); }
};
// the weight that is passed by the last token that top-p keeps
__device__ __forceinline__ u64 passed(float share, u64 all) {
    const double below = ceil((double)share * (double)all) - 1;
    return below > 0 && all ? min((u64)below, all - 1) : 0;
}
// the bins that a thread adds up
struct Filled {
    u64 mass[2];
    u32 count[2];
};
template <int THREADS>
__device__ __forceinline__ Filled filled_of(const Sample &a, int row) {
    static_assert(2 * THREADS >= kBins);
    Filled f;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int i = 2 * (int)threadIdx.x + k;
        f.mass[k] = i < kBins ? a.ws.mass[(long)row * kBins + i] : 0, f.count[k] = i < kBins ? a.ws.count[(long)row * kBins + i] : 0;
    }
    return f;
}
template <int THREADS>
__device__ Cut cut_of(const Row &r, const Filled &filled, Bins &bins) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    constexpr int kEach = 2;
    u64 m[kEach], sum = 0;
    u32 n[kEach], all = 0;
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        sum += filled.mass[k], all += filled.count[k];
        m[k] = sum, n[k] = all;
    }
    u64 before = upto_of(sum);
    u32 count = (u32)upto_of(all);
    if (lane == 63) bins.part_mass[wave] = before, bins.part_count[wave] = count;
    if (tid == 0) bins.k_bin = kBins - 1, bins.p_low = bins.p_high = kBins - 1;
    __syncthreads();
    before -= sum, count -= all;
    for (int k = 0; k < wave; ++k) before += bins.part_mass[k], count += bins.part_count[k];
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const int i = tid * kEach + k;
        if (i >= kBins) continue;
        bins.mass[i] = before + m[k], bins.count[i] = count + n[k];
        if (r.most > 0 && i < kBins - 1 && count + n[k] >= (u32)r.most && count + (k ? n[k - 1] : 0) < (u32)r.most) bins.k_bin = i;
    }
    __syncthreads();
    Cut c;
    c.k_bin = bins.k_bin, c.by_k = r.most > 0 && c.k_bin < kBins - 1;
    c.low = kBins, c.high = -1;
    c.sure = c.by_k ? c.k_bin : kBins;
    if (r.share < 1) {
        // what top-p takes its share of lies between these, and so do the bins of its cut
        const u64 total = bins.mass[kBins - 1];
        const u64 low = passed(r.share, c.by_k ? (c.k_bin ? bins.mass[c.k_bin - 1] : 0) : total), high = passed(r.share, c.by_k ? bins.mass[c.k_bin] : total);
        for (int i = tid; i < kBins; i += THREADS) {
            const u64 at = i ? bins.mass[i - 1] : 0;
            if (at <= low && low < bins.mass[i]) bins.p_low = i;
            if (at <= high && high < bins.mass[i]) bins.p_high = i;
        }
        __syncthreads();
        c.low = min(bins.p_low, c.k_bin), c.high = min(bins.p_high, c.k_bin), c.sure = c.low;
    }
    return c;
}

template <int TYPE>
__global__ __launch_bounds__(kThreads) void sample_gather_kernel(Sample a) {
    __shared__ Bins bins;
    __shared__ u64 sure[kMostChunks];
    const int row = blockIdx.x / a.groups, group = blockIdx.x % a.groups, tid = threadIdx.x;
    const int first = group * a.each, chunks = min(a.each, a.chunks - first);
    Logits<TYPE, kThreads> logits(a.logits, row, a.from<TYPE>(row, first), a.from<TYPE>(row, first + chunks));
    const Filled filled = filled_of<kThreads>(a, row);
    const Row r = row_of(a, row);
    if (r.greedy || r.first < 0) return;
    for (int i = tid; i < chunks; i += kThreads) sure[i] = 0;
    Cut cut{kBins, kBins, -1, kBins - 1, false};
    if (r.cuts()) cut = cut_of<kThreads>(r, filled, bins);
    __syncthreads();
    // tokens beyond this bin weigh nothing or less than min-p asks: their weights need not be computed
    const int reach = min(cut.sure, r.least > 0 ? (int)fminf(-logf(r.least) * kBinsPerUnit + 2, kBins - 1) + 1 : kBins - 1);
    const int lo = a.from<TYPE>(row, first), past = chunks > 1 ? a.from<TYPE>(row, first + 1) - a.chunk : lo;
    u64 sum = 0;
    logits.each(
        [&](float z, int i) {
            const int bin = r.bin(z);
            if (bin < reach) sum += r.kept(z);
            if (cut.open(bin)) {
                const u32 at = atomicAdd(&a.ws.listed[row], 1u);
                if (at < kListed) a.ws.list[(long)row * kListed + at] = key_of(z, i);
            }
        },
        [&](int i, int next) {
            const int c = min(max(i - past, 0) >> a.shift, chunks - 1);
            if (next >= 0 && min(max(next - past, 0) >> a.shift, chunks - 1) == c) return;
            sum = wave_sum(sum);
            if ((tid & 63) == 0 && sum) atomicAdd((unsigned long long *)&sure[c], (unsigned long long)sum);
            sum = 0;
        });
    __syncthreads();
    for (int i = tid; i < chunks; i += kThreads) a.ws.sure[(long)row * a.chunks + first + i] = sure[i];
}

struct Search {
    u64 bins[256];
    u64 carry, total;
    u32 digit;
};
// Of elements with keys and weights, given by each(f(key, weight)) over all threads together, the key at which the
// weights added up in ascending order of keys first exceed `target`: digit by digit from the top, in sums of the
// weights of all elements whose digits so far are the key's.  Needs target < the sum of all.
template <class E>
__device__ u64 weighted_select(Search &sh, u64 target, E each) {
    u64 prefix = 0;
    for (int shift = 56; shift >= 0; shift -= 8) {
        for (int i = threadIdx.x; i < 256; i += kDrawThreads) sh.bins[i] = 0;
        __syncthreads();
        each([&](u64 key, u64 weight) {
            if (weight && (shift == 56 || key >> (shift + 8) == prefix >> (shift + 8)))
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

template <int TYPE>
__global__ __launch_bounds__(kDrawThreads) void sample_draw_kernel(Sample a) {
    constexpr int kWaves = kDrawThreads / 64;
    __shared__ Bins bins;
    __shared__ union {
        Search search;
        u64 keys[kListed];
    } sh;
    __shared__ u64 chunk_mass[kMostChunks], part[kWaves], found_mass, found_key;
    __shared__ u64 unsorted[kCounted];
    __shared__ int found, place[kCounted];
    const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // all that does not depend on the cut is asked for at once
    static_assert(kMostChunks <= kDrawThreads);
    const float u = a.how.u[row];
    const u64 sure = tid < a.chunks ? a.ws.sure[(long)row * a.chunks + tid] : 0;
    const int n = (int)a.ws.listed[row];
    const u64 *list = a.ws.list + (long)row * kListed;
    const u64 early = list[tid % kCounted];
    const Filled filled = filled_of<kDrawThreads>(a, row);
    const Row r = row_of(a, row);
    if (r.greedy || r.first < 0) {
        if (tid == 0) a.tokens[row] = r.first;
        return;
    }
    // of a token's index: what its chunks' borders lie behind multiples of a chunk
    const int past = a.chunks > 1 ? a.from<TYPE>(row, 1) - a.chunk : 0;
    if (tid < a.chunks) chunk_mass[tid] = sure;
    // sum over the workgroup's threads
    auto sum_of = [&](u64 v) {
        v = wave_sum(v);
        __syncthreads();
        if (lane == 0) part[wave] = v;
        __syncthreads();
        return wave_sum(lane < kWaves ? part[lane] : 0);
    };
    auto before_wave = [&]() { return wave_sum(lane < wave ? part[lane] : 0); };
    u64 last = ~0ull;                                  // the last key that is kept
    if (r.cuts()) {
        const Cut cut = cut_of<kDrawThreads>(r, filled, bins);
        if (n > kListed) {
            // more than a list holds: the cuts from the whole row, and the chunks' sums anew
            auto each_of = [&](auto weight) {
                return [&a, row, weight, &last](auto f) {
                    Logits<TYPE, kDrawThreads>(a.logits, row, 0, a.vocab).each([&](float z, int i) {
                        const u64 key = key_of(z, i);
                        if (key <= last) f(key, weight(z));
                    });
                };
            };
            auto one = [](float) { return (u64)1; };
            auto weight = [&](float z) { return r.weight(z); };
            if (r.most > 0) last = weighted_select(sh.search, r.most - 1, each_of(one));
            if (r.share < 1) {
                u64 sum = 0;
                each_of(weight)([&](u64, u64 w) { sum += w; });
                last = weighted_select(sh.search, passed(r.share, sum_of(sum)), each_of(weight));
            }
            for (int c = wave; c < a.chunks; c += kWaves) {
                u64 sum = 0;
                for (int i = a.from<TYPE>(row, c) + lane; i < a.from<TYPE>(row, c + 1); i += 64) {
                    const float z = load_value<TYPE>(a.logits, row, i);
                    if (key_of(z, i) <= last) sum += r.kept(z);
                }
                sum = wave_sum(sum);
                if (lane == 0) chunk_mass[c] = sum;
            }
            __syncthreads();
        } else {
            if (n <= kCounted) {
                // a short list in order: a token's place is the number of those before it
                constexpr int kParts = kDrawThreads / kCounted;
                const int c = tid % kCounted;
                if (tid < kCounted) unsorted[tid] = tid < n ? early : ~0ull, place[tid] = 0;
                __syncthreads();
                const u64 own = unsorted[c];
                int before = 0;
#pragma unroll 8
                for (int i = tid / kCounted; i < n; i += kParts) before += unsorted[i] < own;
                if (before) atomicAdd(&place[c], before);
                __syncthreads();
                if (tid < n) sh.keys[place[c]] = own;
            } else {
                int size = 2 * kCounted;
                while (size < n) size *= 2;
                for (int i = tid; i < size; i += kDrawThreads) sh.keys[i] = i < n ? list[i] : ~0ull;
                // a bitonic network
                for (int run = 2; run <= size; run *= 2)
                    for (int step = run / 2; step; step /= 2) {
                        __syncthreads();
                        for (int p = tid; p < size / 2; p += kDrawThreads) {
                            const int i = (p / step) * 2 * step + p % step, j = i + step;
                            const u64 x = sh.keys[i], y = sh.keys[j];
                            if ((x > y) == !(i & run)) sh.keys[i] = y, sh.keys[j] = x;
                        }
                    }
            }
            __syncthreads();
            // neighbours of the list by a thread: their bins, weights, and the weight of the list before them
            constexpr int kOwn = kListed / kDrawThreads;
            u64 key[kOwn], w[kOwn];
            int bin[kOwn];
#pragma unroll
            for (int k = 0; k < kOwn; ++k) {
                const int i = kOwn * tid + k;
                key[k] = i < n ? sh.keys[i] : ~0ull;
                const float z = i < n ? logit_of(key[k]) : 0.0f;
                bin[k] = i < n ? r.bin(z) : kBins;
                w[k] = i < n ? r.weight(z) : 0;
            }
            u64 all = bins.mass[kBins - 1];
            int below = 0;
            if (cut.by_k) {
                // of k_bin's tokens the first ones; other bins' come before them in the list
                const int need = r.most - (cut.k_bin ? (int)bins.count[cut.k_bin - 1] : 0);
                u64 at = 0;
                for (int k = 0; k < kOwn; ++k) at += bin[k] < cut.k_bin;
                below = (int)sum_of(at);
                last = sh.keys[below + need - 1];
                u64 mine = 0;
                for (int k = 0; k < kOwn; ++k) mine += bin[k] == cut.k_bin && key[k] <= last ? w[k] : 0;
                all = (cut.k_bin ? bins.mass[cut.k_bin - 1] : 0) + sum_of(mine);
            }
            if (r.share < 1) {
                const u64 target = passed(r.share, all);
                if (tid == 0) found = kBins - 1;
                __syncthreads();
                for (int i = tid; i < kBins; i += kDrawThreads)
                    if ((i ? bins.mass[i - 1] : 0) <= target && target < bins.mass[i]) found = i;
                __syncthreads();
                const int p_bin = found;
                const u64 rest = target - (p_bin ? bins.mass[p_bin - 1] : 0);
                u64 mine = 0;
                for (int k = 0; k < kOwn; ++k) mine += bin[k] == p_bin ? w[k] : 0;
                const u64 upto = upto_of(mine);
                __syncthreads();
                if (lane == 63) part[wave] = upto;
                __syncthreads();
                u64 at = upto - mine + before_wave();
                for (int k = 0; k < kOwn; ++k) {
                    const u64 own = bin[k] == p_bin ? w[k] : 0;
                    if (at <= rest && rest < at + own) found_key = key[k];
                    at += own;
                }
                __syncthreads();
                last = min(last, found_key);
            }
            // what the list adds to the chunks
            for (int k = 0; k < kOwn; ++k)
                if (key[k] <= last && kOwn * tid + k < n && bin[k] >= cut.sure) {
                    const u64 kept = r.kept(logit_of(key[k]));
                    if (kept) atomicAdd((unsigned long long *)&chunk_mass[min(max((int)(u32)key[k] - past, 0) >> a.shift, a.chunks - 1)], (unsigned long long)kept);
                }
            __syncthreads();
        }
    } else {
        __syncthreads();
    }
    // the chunk, then the token
    u64 sum = 0;
    for (int i = tid; i < a.chunks; i += kDrawThreads) sum += chunk_mass[i];
    if (tid == 0) found = 0, found_mass = 0;
    const u64 all = sum_of(sum);
    const double drawn = (double)u * (double)all;
    u64 target = drawn > 0 ? min((u64)drawn, all - 1) : 0;
    if (wave == 0) {
        constexpr int kOf = kMostChunks / 64;
        u64 own[kOf], mine = 0;
        for (int k = 0; k < kOf; ++k) mine += own[k] = lane * kOf + k < a.chunks ? chunk_mass[lane * kOf + k] : 0;
        u64 at = upto_of(mine) - mine;
        for (int k = 0; k < kOf; ++k) {
            if (at <= target && target < at + own[k]) found = lane * kOf + k, found_mass = target - at;
            at += own[k];
        }
    }
    __syncthreads();
    target = found_mass;
    // the chunk's tokens in runs of a thread each, all of them at once where a chunk is as usual
    constexpr int kRun = 8;
    const int hi = a.from<TYPE>(row, found + 1);
    for (int lo = a.from<TYPE>(row, found); lo < hi; lo += kRun * kDrawThreads) {
        float z[kRun];
        u64 w[kRun], mine = 0;
#pragma unroll
        for (int k = 0; k < kRun; ++k) z[k] = load_value<TYPE>(a.logits, row, min(lo + tid * kRun + k, hi - 1));
#pragma unroll
        for (int k = 0; k < kRun; ++k) {
            const int i = lo + tid * kRun + k;
            mine += w[k] = i < hi && key_of(z[k], i) <= last ? r.kept(z[k]) : 0;
        }
        const u64 upto = upto_of(mine);
        __syncthreads();
        if (lane == 63) part[wave] = upto;
        __syncthreads();
        u64 at = before_wave() + upto - mine;
        if (at <= target && target < at + mine)
            for (int k = 0; k < kRun; ++k) {
                if (at <= target && target < at + w[k]) a.tokens[row] = lo + tid * kRun + k;
                at += w[k];
            }
        const u64 run = wave_sum(lane < kWaves ? part[lane] : 0);
        if (target < run) break;
        target -= run;
    }
}

// Chunks of a row: 2048 tokens, which the last launch goes through for the token; more where a row would have too many
// (64 rows of 100003 logits 36.1 us with 2048, 38.8 with 4096, 36.3 with 1024; 256 of 131072 residues 118, 117 and 126).
// Workgroups of a row: enough for the card, with whole chunks each; 640 of all rows take 113 us for those residues, 512 118.
void cut_up(Sample &a) {
    a.shift = 11;
    while (((long)a.vocab + (1l << a.shift) - 1) >> a.shift > kMostChunks) ++a.shift;
    a.chunk = 1 << a.shift;
    a.chunks = (int)(((long)a.vocab + a.chunk - 1) / a.chunk);
    const int wanted = std::max(1, std::min(a.chunks, (640 + a.rows - 1) / std::max(a.rows, 1)));
    a.each = (a.chunks + wanted - 1) / wanted;
    a.groups = (a.chunks + a.each - 1) / a.each;
}

}  // namespace

namespace gala {

size_t sample_workspace(int rows, int vocab) {
    Sample a{};
    a.rows = rows, a.vocab = vocab;
    cut_up(a);
    return (size_t)rows * (kBins * 12 + kListed * 8 + (a.chunks + a.groups) * 8 + 8);
}

int launch_sample(void *stream, const Values &logits, int rows, int vocab, const gala_sampling &how, int *tokens, void *workspace) {
    Sample a{};
    a.logits = logits, a.rows = rows, a.vocab = vocab, a.how = how, a.tokens = tokens;
    cut_up(a);
    u64 *at = (u64 *)workspace;
    a.ws.mass = at, at += (size_t)rows * kBins;
    a.ws.list = at, at += (size_t)rows * kListed;
    a.ws.best = at, at += (size_t)rows * a.groups;
    a.ws.sure = at, at += (size_t)rows * a.chunks;
    a.ws.count = (u32 *)at;
    a.ws.listed = a.ws.count + (size_t)rows * kBins;
    const dim3 grid(rows * a.groups);
    hipStream_t st = (hipStream_t)stream;
    by_type(logits.type, [&](auto type) {
        constexpr int T = decltype(type)::value;
        hipLaunchKernelGGL(sample_best_kernel<T>, grid, dim3(kThreads), 0, st, a);
        if (how.top_k || how.top_p) hipLaunchKernelGGL(sample_bins_kernel<T>, grid, dim3(kThreads), 0, st, a);
        hipLaunchKernelGGL(sample_gather_kernel<T>, grid, dim3(kThreads), 0, st, a);
        hipLaunchKernelGGL(sample_draw_kernel<T>, dim3(rows), dim3(kDrawThreads), 0, st, a);
    });
    return hipGetLastError() != hipSuccess;
}

}  // namespace gala
