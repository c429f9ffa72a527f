// Attention of a batch's queries over the paged 4-bit cache.
#include "gala_attention.h"
#include "gala_attention4_cut.h"

using namespace gala;

namespace {

typedef __bf16 v8b __attribute__((ext_vector_type(8)));
typedef __bf16 v2b __attribute__((ext_vector_type(2)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));

// A head of G x 32 channels is multiplied in G products of 32.  Four lanes (parts) have a token's key: of four groups of 32
// channels one each, of two left over half a group each, of one left over eight channels each, so that a lane loads 16,
// 8 or 4 bytes.  Product n takes the lanes' n-th words: the order of channels within it is the queries' too.
template <int G>
struct Words {
    static constexpr int kFours = G / 4;
    // group and word within it
    static __device__ __forceinline__ int group(int n, int part) {
        if (n < 4 * kFours) return n / 4 * 4 + part;
        if ((G & 2) && n < 4 * kFours + 2) return 4 * kFours + (part >> 1);
        return G - 1;
    }
    static __device__ __forceinline__ int word(int n, int part) {
        if (n < 4 * kFours) return n & 3;
        if ((G & 2) && n < 4 * kFours + 2) return (part & 1) * 2 + (n & 1);
        return part;
    }
};
template <int G>
struct Keys {
    u32 code[4][G];          // of four tiles of 16 tokens
    u32 exponent[G];         // a byte for each tile; word n's
};
template <int G>
__device__ __forceinline__ void load_keys(const char *data, int token, int part, Keys<G> &k) {
    typedef Words<G> W;
    constexpr int kTwo = 4 * W::kFours;
    auto at = [&](int i, int n) { return data + (i * G + W::group(n, part)) * 256 + token * 16 + W::word(n, part) * 4; };
    auto exponent = [&](int n) { return *(const u32 *)(data + kv4_exponents(G) + token * 4 + W::group(n, part) * 64); };
#pragma unroll
    for (int n = 0; n < kTwo; n += 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int4 x = *(const int4 *)at(i, n);
            k.code[i][n] = x.x, k.code[i][n + 1] = x.y, k.code[i][n + 2] = x.z, k.code[i][n + 3] = x.w;
        }
        k.exponent[n] = k.exponent[n + 1] = k.exponent[n + 2] = k.exponent[n + 3] = exponent(n);
    }
    if constexpr (G & 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int2 x = *(const int2 *)at(i, kTwo);
            k.code[i][kTwo] = x.x, k.code[i][kTwo + 1] = x.y;
        }
        k.exponent[kTwo] = k.exponent[kTwo + 1] = exponent(kTwo);
    }
    if constexpr (G & 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) k.code[i][G - 1] = *(const u32 *)at(i, G - 1);
        k.exponent[G - 1] = exponent(G - 1);
    }
}
__device__ __forceinline__ v8b numbers_of(u32 codes, float scale) {
    union {
        v2b pair[4];
        v8b all;
    } u;
    u.pair[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0);
    u.pair[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
    u.pair[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2);
    u.pair[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
    return u.all;
}
__device__ __forceinline__ v8h halves_of(u32 codes) {
    union {
        v2h pair[4];
        v8h all;
    } u;
    u.pair[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, 1.0f, 0);
    u.pair[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, 1.0f, 1);
    u.pair[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, 1.0f, 2);
    u.pair[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, 1.0f, 3);
    return u.all;
}
// what the byte of tile i stands for
__device__ __forceinline__ float power_of(u32 exponents, int i) {
    return __uint_as_float((i < 3 ? exponents << (24 - 8 * i) >> 1 : exponents >> 1) & 0x7f800000u);
}
// x as the sum of N bfloat16 numbers of eight bits each: the first ones cut off, the last one rounded, so that 8 N bits of x are
// kept, to half a step
template <int N>
__device__ __forceinline__ void parts_of(float (&x)[8], v8b (&to)[N]) {
    union {
        u32 word[4];
        v8b all;
    } u;
#pragma unroll
    for (int n = 0; n + 1 < N; ++n) {
#pragma unroll
        for (int k = 0; k < 4; ++k) u.word[k] = __builtin_amdgcn_perm(__float_as_uint(x[2 * k + 1]), __float_as_uint(x[2 * k]), 0x07060302);
        to[n] = u.all;
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] -= __uint_as_float(__float_as_uint(x[k]) & 0xffff0000u);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) to[N - 1][k] = (__bf16)x[k];
}

// A lane's part of a query in NQ bfloat16 parts, 0 for a number that is none; whether all of it, over the four lanes, are numbers
template <int G, int NQ>
__device__ __forceinline__ bool load_query(const Attention &a, long row, int hq, int part, v8b (&q)[G][NQ]) {
    typedef Words<G> W;
    int fine = 1;
    auto load = [&](auto type) __attribute__((always_inline)) {
#pragma unroll
        for (int n = 0; n < G; ++n) {
            float x[8];
            const int d = W::group(n, part) * 32 + W::word(n, part) * 8;
            load_channels<decltype(type)::value, 1>(a.q, a.pieces, row, hq * a.kv.dim + d, hq * a.kv.dim + a.kv.dim, x);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                fine &= fabsf(x[k]) < INFINITY;
                x[k] = fabsf(x[k]) < INFINITY ? x[k] : 0.0f;
            }
            parts_of<NQ>(x, q[n]);
        }
    };
    by_type(a.q.type, load);
    fine &= __shfl_xor(fine, 16);
    fine &= __shfl_xor(fine, 32);
    return fine;
}

// ---- weights in half precision -------------------------------------------------------------------------------------------
// Of 16-bit types a weight w = p * s, p = exp(score - ...) and s its token's scale of values, comes from one exponential: log2(s) is
// the score's initial value in the accumulators.  It enters the second product in half precision, raised so that the largest is
// between 2^7 and 2^15: 11 bits down to 2^-21 of the largest weight times scale, steps of 2^-31 of it below.  The divisor adds up w / s in
// 32 bits.
// A choice: a weight is off by at most 2^-12 of itself, an eighth of the rounding of a bf16 result, whose distance from the exact one grows
// by less than 1 % (2 x 1000 queries over 2000 tokens: 1.669e-3 root-mean-square, 1.658e-3 rounded from exact ones).  For f16 it is as large
// as the result's rounding: single tokens have a second part (2.09e-4, the rounding alone), prompts, whose registers do not hold one
// beside two parts of the queries (253 of 256 at 128 channels), do not (2.84e-4 instead of 2.08e-4).
constexpr float kRaised = 7, kHighest = 15;      // exponents
constexpr float kNothing = 0x1p-88f;             // scale of values that are zeros: their weights count in the divisor
constexpr float kOrdinary = 0x1p14f;             // up to here and down to kNothing w / s stays within 32 bits where its weight matters

// A wavefront's scales of a block, a token a lane, in LDS: log2(s) / unit and 1 / s.  What is no scale of a number belongs to a token
// that is not seen, or to zeros.
typedef float Scales[2][kKvBlock];
__device__ __forceinline__ void put_scales(Scales &to, int lane, u32 scale, float per_unit) {
    const float given = __uint_as_float(scale << 16), held = given >= 0x1p-100f && given < INFINITY ? given : kNothing;
    to[0][lane] = __builtin_amdgcn_logf(held) * per_unit;
    to[1][lane] = __builtin_amdgcn_rcpf(held);
    __builtin_amdgcn_wave_barrier();                 // a wavefront's own: its instructions on LDS are done in order
}
// Of a block's scales, a token a lane, all that some query of the tile sees: what lies behind a sequence's end, in front of a window or in
// the first page for a missing one may be anything and chooses nothing.  Who sees what is asked where some scale is not ordinary:
// asked of every block it costs prompts 1 to 4 %, so 0 to 2.6 (256 channels).
__device__ __forceinline__ bool ordinary_scales(const Attention &a, const Seen &s, int block, int page, u32 scale) {
    const float x = __uint_as_float(scale << 16);
    const u64 apart = __ballot((x >= 0x1p-100f && x < kNothing) || (x > kOrdinary && x < INFINITY));
    if (__builtin_expect(!apart, 1)) return true;
    const int own = block * kKvBlock, hi = min(s.at_hi + 1, page < 0 ? 0 : a.kv.max_len) - own;
    const int lo = a.window ? s.at_lo - a.window + 1 - own : 0, sinks = a.sinks - own;
    auto below = [](int n) { return n <= 0 ? 0 : n >= 64 ? ~0ull : (1ull << n) - 1; };
    return !(apart & below(hi) & (~below(lo) | below(sinks)));
}
// From a wavefront's first scale on that is not ordinary (bfloat16 alone has such), a lane's divisor is sum * 2^apart with
// the largest weight's exponent for `apart`: weights' own exponents are those of w less log2(s).
template <int N>
__device__ __forceinline__ void add_apart(const float (&x)[N], float &sum, float &apart) {
    float most = sum > 0 ? apart : -INFINITY;
#pragma unroll
    for (int k = 0; k < N; ++k) most = fmaxf(most, x[k]);
    if (most == -INFINITY) return;
    sum = sum > 0 ? sum * __builtin_amdgcn_exp2f(apart - most) : 0.0f;
#pragma unroll
    for (int k = 0; k < N; ++k) sum += __builtin_amdgcn_exp2f(x[k] - most);
    apart = most;
}
// ... and in the end, of lanes with the same column: what the column's sums are multiplied by
__device__ __forceinline__ float joined_apart(int lanes, float &sum, float &apart) {
    float most = sum > 0 ? apart : -INFINITY;
    for (int k = lanes; k < 64; k <<= 1) most = fmaxf(most, __shfl_xor(most, k));
    if (most == -INFINITY) most = 0;
    sum = sum > 0 ? sum * __builtin_amdgcn_exp2f(apart - most) : 0.0f;
    apart = most;
    return __builtin_amdgcn_exp2f(-most);
}
// where the scale of a lane's token lies
template <int G>
__device__ __forceinline__ int scale_place(int lane) { return kv4_scales(G) + (lane % 16 / 4 * 16 + lane / 16 * 4 + lane % 4) * 2; }
// exponents of a column that the base is taken off already; other lanes with the same column are `lanes` and more apart
template <int N, int M, class V, class O>
__device__ __forceinline__ void raise_base(V (&x)[N], float most, int lanes, const bool ordinary, float &base, float &limit, float &sum, float &apart, O (&o)[M]) {
    if (!__any(most > limit)) return;
    for (int k = lanes; k < 64; k <<= 1) most = fmaxf(most, __shfl_xor(most, k));
    if (most > limit || most > kRaised) {
        most -= kRaised;
        const float was = limit == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(-most);          // nothing yet with the first base
        base += most;
        limit = kHighest;
        if (ordinary)
            sum *= was;
        else
            apart -= most;
#pragma unroll
        for (int j = 0; j < M; ++j) o[j] *= was;
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] -= most;
    }
}

// Scores are products of the codes with their powers of two, exact in bfloat16, and of the queries in NQ bfloat16 parts (8 bits
// each; a query of 8, 11 or 24 bits is all of its parts).  Of a block's scores a lane has 16 of one column's, and they are
// the very weights that it hands to the second product, because the values' codes lie in that order of tokens: a block goes from memory
// to the sums without LDS or an exchange between lanes, but for the largest score.  FINE: a weight takes its token's scale of
// values along and is cut into three bfloat16 parts, 24 bits; else as above, where f16 comes in or out in two parts, 22 bits: one
// rounding of a weight is as large as that of an f16 result, and few keys do not average it out.  A wavefront has blocks of its
// own; a workgroup's wavefronts are joined at the end.
// Bound by HBM where the cache is large (64 queries of up to 8192 tokens, 424 MB: 86 us, 4.9 TB/s; 131072 tokens, 70 MB: 22 us
// with 5 for the join, 24 where none of it is in the last-level cache), by a chain of starts, table, codes where it is not (1000 tokens 8 us).  Products of 16 x 16: of few queries most
// columns are empty, and a tile of 32 would have twice as many.
template <int G, int NQ, bool FINE, int kWaves>
__global__ __launch_bounds__(64 * kWaves, G <= 4 ? 2 : 1) void kv4_attention_kernel(Attention a) {
    constexpr int NV = 2 * G;                                // tiles of 16 channels of values
    constexpr int kParts = NQ == 2 ? 2 : 1;                  // of a weight in half precision
    constexpr size_t kHead = 64 * (33 * G + 2);
    constexpr int kRow = NV * 16 + 1;
    extern __shared__ float sums[];                          // of each wavefront and column
    __shared__ float stats[kWaves][kColumns][2];
    __shared__ __attribute__((aligned(16))) Scales of_scales[FINE ? 1 : kWaves];
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
    // The next block's keys are under way while this one's weights are made, the one after's page too.
    Keys<G> keys;
    u32 scale = 0;
    int u = from + wave, page, page_next;
    auto page_at = [&](int v) { return v < to ? page_of(kv, b, s.block(v)) : -1; };
    // without a page the first one is read and not seen: no branch around what is under way
    auto data_of = [&](int page) { return (const char *)kv.codes + ((size_t)max(page, 0) * kv.heads + h) * kHead; };
    auto load = [&](int page) __attribute__((always_inline)) {
        const char *data = data_of(page);
        load_keys<G>(data, col, part, keys);
        if constexpr (!FINE) scale = *(const unsigned short *)(data + scale_place<G>(lane));
    };
    page = page_at(u), page_next = page_at(u + kWaves);
    if (u < to) load(page);
    // the column's query
    const int c = s.col0 + min(col, s.cols - 1), qi = c / a.group, g = c % a.group;
    const long row = s.start + qi;
    const int at = s.at_lo - s.col0 / a.group + qi, hq = h * a.group + g;
    v8b q[G][NQ];
    const bool bad = !load_query<G, NQ>(a, row, hq, part, q);
    const float unit_q = a.scale * kLog2E, per_unit = FINE ? 0.0f : 1.0f / unit_q;
    v4f o[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) o[j] = v4f{0, 0, 0, 0};
    // FINE: the base is the largest score; else limit is what an exponent may be before the base is raised
    float base = FINE ? -INFINITY : 0, limit = -INFINITY, sum = 0, apart = 0;
    auto step = [&](auto all_ordinary) __attribute__((always_inline)) {
        constexpr bool ordinary = decltype(all_ordinary)::value;
        const int block = s.block(u), end = page < 0 ? 0 : kv.max_len;
        const char *data = data_of(page);
        u32 values[G][4];
#pragma unroll
        for (int j = 0; j < G; ++j) {
            const int4 x = *(const int4 *)(data + 1024 * G + j * 1024 + lane * 16);
            values[j][0] = x.x, values[j][1] = x.y, values[j][2] = x.z, values[j][3] = x.w;
        }
        v4f scale_v[4];          // FINE: the scales; else their reciprocals
        if constexpr (FINE) {
            const int4 *from = (const int4 *)(data + kv4_scales(G) + part * 32);
            const int4 x = from[0], y = from[1];
            const u32 w[8] = {(u32)x.x, (u32)x.y, (u32)x.z, (u32)x.w, (u32)y.x, (u32)y.y, (u32)y.z, (u32)y.w};
#pragma unroll
            for (int k = 0; k < 16; ++k) scale_v[k / 4][k % 4] = __uint_as_float(k & 1 ? w[k / 2] & 0xffff0000u : w[k / 2] << 16);
        } else {
            if (ordinary && !ordinary_scales(a, s, block, page, scale)) return false;
            put_scales(of_scales[wave], lane, scale, per_unit);
        }
        v4f t[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (FINE)
                t[i] = v4f{0, 0, 0, 0};
            else
                t[i] = *(const v4f *)&of_scales[wave][0][i * 16 + part * 4];
            v8b k[G];
#pragma unroll
            for (int n = 0; n < G; ++n) k[n] = numbers_of(keys.code[i][n], power_of(keys.exponent[n], i));
#pragma unroll
            for (int p = NQ - 1; p >= 0; --p)        // the small parts first
#pragma unroll
                for (int n = 0; n < G; ++n) t[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[n], q[n][p], t[i], 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; ++r) t[i][r] = FINE ? t[i][r] * unit_q : fmaf(t[i][r], unit_q, -base);
        }
        if constexpr (!FINE) {
#pragma unroll
            for (int i = 0; i < 4; ++i) scale_v[i] = *(const v4f *)&of_scales[wave][1][i * 16 + part * 4];
        }
        page = page_next;
        load(page);
        page_next = page_at(u + 2 * kWaves);
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
                    const bool seen = (e <= hi) & ((e >= lo) | (e < sinks));
                    t[i][r] = seen ? t[i][r] : -INFINITY;
                    if constexpr (FINE) scale_v[i][r] = seen ? scale_v[i][r] : 0.0f;           // what is not seen may be no number
                }
        }
        float most = t[0][0];
#pragma unroll
        for (int i = 1; i < 16; ++i) most = fmaxf(most, t[i / 4][i % 4]);
        if constexpr (FINE) {
            most = fmaxf(most, __shfl_xor(most, 16));
            most = fmaxf(most, __shfl_xor(most, 32));
            if (__any(most > base)) {
                const float now = fmaxf(base, most), was = now > base ? __builtin_amdgcn_exp2f(base - now) : 1.0f;
                base = now;
                sum *= was;
#pragma unroll
                for (int j = 0; j < NV; ++j) o[j] *= was;
            }
            const float off = base == -INFINITY ? 0.0f : base;
            v8b w[2][3];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                float x[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float p = __builtin_amdgcn_exp2f(t[2 * half + k / 4][k % 4] - off);
                    sum += p;
                    x[k] = p * scale_v[2 * half + k / 4][k % 4];
                }
                parts_of<3>(x, w[half]);
            }
#pragma unroll
            for (int j = 0; j < NV; ++j) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const v8b v = numbers_of(values[j >> 1][(j & 1) * 2 + half], 1.0f);
#pragma unroll
                    for (int p = 2; p >= 0; --p) o[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, w[half][p], o[j], 0, 0, 0);
                }
            }
        } else {
            raise_base(t, most, 16, ordinary, base, limit, sum, apart, o);
            if (!ordinary) {
                float x[16];
#pragma unroll
                for (int k = 0; k < 16; ++k) x[k] = fmaf(-of_scales[wave][0][k / 4 * 16 + part * 4 + k % 4], unit_q, t[k / 4][k % 4]);
                add_apart(x, sum, apart);
            }
            float added = 0;
            v8h w[2][kParts];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float x = __builtin_amdgcn_exp2f(t[i][r]);
                    added = fmaf(x, scale_v[i][r], added);
                    const _Float16 first = (_Float16)x;
                    w[i >> 1][0][(i & 1) * 4 + r] = first;
                    if constexpr (kParts == 2) w[i >> 1][1][(i & 1) * 4 + r] = (_Float16)(x - (float)first);
                }
            if (ordinary) sum += added;
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    const v8h v = halves_of(values[j >> 1][(j & 1) * 2 + half]);
#pragma unroll
                    for (int p = kParts - 1; p >= 0; --p) o[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, w[half][p], o[j], 0, 0, 0);
                }
        }
        return true;
    };
    for (; u < to && step(std::true_type()); u += kWaves) {}
    const bool ordinary = FINE || u >= to;
    if constexpr (!FINE)
        for (; u < to; u += kWaves) step(std::false_type());
    // the wavefronts' sums in one
    if (!ordinary) {
        const float f = joined_apart(16, sum, apart);
        base += apart;
#pragma unroll
        for (int j = 0; j < NV; ++j) o[j] *= f;
    }
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (!FINE && limit == -INFINITY) base = -INFINITY;
    if (col < a.columns) {
        float *mine = sums + (wave * a.columns + col) * kRow + part * 4;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) mine[j * 16 + r] = o[j][r];
    }
    if (part == 0) stats[wave][col][0] = bad ? __builtin_nanf("") : base, stats[wave][col][1] = sum;
    __syncthreads();
    const long place = (((long)b * kv.heads + h) * a.tiles + tile) * a.splits + split;
    for (int e = threadIdx.x; e < s.cols * kv.dim; e += 64 * kWaves) {
        const int cc = e / kv.dim, d = e % kv.dim;
        float most = -INFINITY, all = 0, x = 0;
#pragma unroll
        for (int k = 0; k < kWaves; ++k) most = fmaxf(most, stats[k][cc][0]);
        const float off = most == -INFINITY ? 0.0f : most;
#pragma unroll
        for (int k = 0; k < kWaves; ++k) {
            const float f = __builtin_amdgcn_exp2f(stats[k][cc][0] - off);       // NaN where the query is
            all += f * stats[k][cc][1];
            x += f * sums[(k * a.columns + cc) * kRow + d];
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

// ---- many queries of a sequence ---------------------------------------------------------------------------------------
// A wavefront has 32 queries for all the keys that they see, in products of 32 x 32: those of 16 x 16 reach 0.7 of their rate, and
// leave less room for the vector ALU between them (23 cycles for half the work, 31 with four multiply-adds; 33 and 35).
// Keys and values come to the registers straight from memory: through LDS they are loaded once a workgroup, but its wavefronts wait for
// each other (4 x 4096 queries over 8192 tokens 1671 us against 1600).  Bound by the vector ALU (0.57 of the SIMDs' cycles) and the products
// (0.38), which the two wavefronts of a SIMD overlap little: 2000 and 1258 queries over 5207 and 3276 tokens, 192 G of operations, 216 us
// (241 from idle clocks), 0.89 P a second, 4 x 4096 over 8192 1.01.
// Two lanes (halves) have a token's key: of two groups of 32 channels one each, of one left over half.  Product n takes their n-th words.
template <int G>
struct WideWords {
    static constexpr int kTwos = G / 2;
    static __device__ __forceinline__ int group(int n, int half) { return n < 4 * kTwos ? n / 4 * 2 + half : G - 1; }
    static __device__ __forceinline__ int word(int n, int half) { return n < 4 * kTwos ? n & 3 : 2 * half + (n & 1); }
};
template <int G>
struct WideKeys {
    u32 code[2][2 * G];              // of two tiles of 32 tokens
    u32 exponent[(G + 1) / 2];       // bytes of all tiles of 16
};
template <int G>
__device__ __forceinline__ void load_keys(const char *data, int token, int half, WideKeys<G> &k) {
    typedef WideWords<G> W;
    const int low = token & 15, high = token >> 4;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const char *tile = data + (2 * i + high) * G * 256 + low * 16;
#pragma unroll
        for (int n = 0; n < 4 * W::kTwos; n += 4) {
            const int4 x = *(const int4 *)(tile + W::group(n, half) * 256);
            k.code[i][n] = x.x, k.code[i][n + 1] = x.y, k.code[i][n + 2] = x.z, k.code[i][n + 3] = x.w;
        }
        if constexpr (G & 1) {
            const int2 x = *(const int2 *)(tile + (G - 1) * 256 + half * 8);
            k.code[i][2 * G - 2] = x.x, k.code[i][2 * G - 1] = x.y;
        }
    }
#pragma unroll
    for (int n = 0; n < (G + 1) / 2; ++n)         // the wanted bytes: the first, and the third for the second tile
        k.exponent[n] = *(const u32 *)(data + kv4_exponents(G) + W::group(4 * n, half) * 64 + low * 4) >> 8 * high & 0xff00ffu;
}

// groups of kColumnsOf queries of a head of sequence b, and how many groups' positions it is shorter than max_len
__device__ __forceinline__ int groups_of(const Attention &a, int b) {
    const int n = min(a.kv.starts[b + 1] - a.kv.starts[b], a.kv.max_new);
    return n > 0 ? (int)(((long)n * a.group + kColumnsOf - 1) / kColumnsOf) : 0;
}
__device__ __forceinline__ int later_of(const Attention &a, int b) {
    return (int)min((long)max(a.kv.max_len - a.kv.lens[b], 0) * a.group / kColumnsOf, (long)a.tiles);
}
// The unit'th group of queries by level, of up to 64 sequences, one a lane: (sequence, group of it), group -1 for none.  Groups are
// packed: workgroups with nothing to do between the others would leave their CUs with less than the rest.
__device__ __forceinline__ int2 ordered(const Attention &a, int unit) {
    const int lane = threadIdx.x & 63, mine = min(lane, a.kv.count - 1);
    const int groups = lane < a.kv.count ? groups_of(a, mine) : 0, later = later_of(a, mine);
    const int width = a.kv.count > 1 ? 64 >> __clz(a.kv.count - 1) - 26 : 1;             // lanes that have one
    // groups before a level; the last level with at most `unit` of them
    auto before = [&](int level) {
        int n = min(max(level - later, 0), groups);
        for (int k = width / 2; k; k >>= 1) n += __shfl_xor(n, k);
        return __builtin_amdgcn_readfirstlane(n);
    };
    int lo = 0, hi = 2 * a.tiles;
    if (before(hi) <= unit) return int2{0, -1};
    while (lo + 1 < hi) {
        const int mid = (lo + hi) >> 1;
        (before(mid) <= unit ? lo : hi) = mid;
    }
    u64 there = __ballot(lo >= later && lo - later < groups);
    for (int k = unit - before(lo); k > 0; --k) there &= there - 1;
    const int b = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)there) - 1);
    return int2{b, __builtin_amdgcn_readlane(groups - 1 - (lo - later), b)};
}

template <int G, int NQ>
__global__ __launch_bounds__(64 * kWavesOf, G <= 4 ? 2 : 1) void kv4_attention_many_kernel(Attention a) {
    typedef float v16f __attribute__((ext_vector_type(16)));
    typedef WideWords<G> W;
    constexpr size_t kHead = 64 * (33 * G + 2);
    __shared__ __attribute__((aligned(16))) Scales of_scales[kWavesOf];
    const KvArgs &kv = a.kv;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
    // Groups of queries that see most keys go first, of all sequences and heads.  A level is that many positions as a group has; a
    // sequence's last group is at the level of its distance from max_len.
    const int h = blockIdx.x % kv.heads, b0 = blockIdx.x / kv.heads;
    const int2 of = a.ordered ? ordered(a, b0) : int2{b0 % kv.count, groups_of(a, b0 % kv.count) - 1 - b0 / kv.count};
    const int b = of.x, group = of.y;
    if (group < 0) return;
    const Seen s = seen_by(a, b, group * kWavesOf + wave, kWide);
    if (!s.cols) return;
    const int mine = s.col0 + min(col, s.cols - 1), qi = mine / a.group;
    const int at = s.at_lo - s.col0 / a.group + qi;
    v8b q[2 * G][NQ];
    u64 bad;                                 // a bit a lane
    {
        const int hq = h * a.group + mine % a.group;
        const long row = s.start + qi;
        int fine = 1;
        auto load = [&](auto type) __attribute__((always_inline)) {
#pragma unroll
            for (int n = 0; n < 2 * G; ++n) {
                float x[8];
                load_channels<decltype(type)::value, 1>(a.q, a.pieces, row, hq * kv.dim + W::group(n, half) * 32 + W::word(n, half) * 8, hq * kv.dim + kv.dim, x);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    fine &= fabsf(x[k]) < INFINITY;
                    x[k] = fabsf(x[k]) < INFINITY ? x[k] : 0.0f;
                }
                parts_of<NQ>(x, q[n]);
            }
        };
        if (a.q.type == GALA_F16)
            load(std::integral_constant<int, GALA_F16>());
        else
            load(std::integral_constant<int, GALA_BF16>());
        fine &= __shfl_xor(fine, 32);
        bad = __ballot(!fine);
    }
    const float unit_q = a.scale * kLog2E, per_unit = 1.0f / unit_q;
    v16f o[G];
    float base = 0, limit = -INFINITY, sum = 0, apart = 0;       // limit: what an exponent may be before the base is raised
#pragma unroll
    for (int j = 0; j < G; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[j][r] = 0;
    WideKeys<G> keys;
    u32 scale;
    auto page_at = [&](int u) { return u < s.total ? page_of(kv, b, s.block(u)) : -1; };
    // without a page the first one is read and not seen: no branch around what is under way
    auto data_of = [&](int page) { return (const char *)kv.codes + ((size_t)max(page, 0) * kv.heads + h) * kHead; };
    auto load = [&](int page) __attribute__((always_inline)) {
        const char *data = data_of(page);
        load_keys<G>(data, col, half, keys);
        scale = *(const unsigned short *)(data + scale_place<G>(lane));
    };
    int page = page_at(0), page_next = page_at(1);
    if (s.total) load(page);
    // Two loops: a branch among the weights costs heads of 128 channels 1 %, of 64 and 256 5 %
    int u = 0;
    auto step = [&](auto ordinary) __attribute__((always_inline)) {
        const int block = s.block(u), end = page < 0 ? 0 : kv.max_len, t0 = block * kKvBlock;
        const char *data = data_of(page);
        if (!ordinary) load(page);               // no registers for the next one's
        // of 16 tokens that a lane's scores of a tile are: those of the first and third four, of the second and fourth
        u32 values[G][2][2];
#pragma unroll
        for (int j = 0; j < G; ++j)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int2 x = *(const int2 *)(data + 1024 * G + j * 1024 + ((half + 2 * k) * 16 + (col & 15)) * 16 + (col >> 4) * 8);
                values[j][0][k] = x.x, values[j][1][k] = x.y;
            }
        put_scales(of_scales[wave], lane, scale, per_unit);
        v16f acc[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const v4f x = *(const v4f *)&of_scales[wave][0][i * 32 + k * 8 + half * 4];
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[i][4 * k + r] = x[r];
            }
        }
#pragma unroll
        for (int n = 0; n < 2 * G; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const u32 e = keys.exponent[n < 4 * W::kTwos ? n / 4 : W::kTwos];
                const v8b k = numbers_of(keys.code[i][n], __uint_as_float(i ? e << 7 & 0x7f800000u : e << 23));
#pragma unroll
                for (int p = NQ - 1; p >= 0; --p) acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q[n][p], acc[i], 0, 0, 0);
            }
        page = page_next;
        if (ordinary) load(page);
        page_next = page_at(u + 2);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][r] = fmaf(acc[i][r], unit_q, -base);
        if (t0 + 63 > s.at_lo || t0 + 64 > end || (a.window && t0 <= s.at_hi - a.window)) {
            const int own = t0 + half * 4, hi = min(at, end - 1) - own;
            const int lo = a.window ? at - a.window + 1 - own : -kKvBlock, sinks = a.window ? a.sinks - own : 0;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int e = i * 32 + r / 4 * 8 + r % 4;
                    acc[i][r] = (e <= hi) & ((e >= lo) | (e < sinks)) ? acc[i][r] : -INFINITY;
                }
        }
        float most = -INFINITY;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) most = fmaxf(most, acc[i][r]);
        raise_base(acc, most, 32, ordinary, base, limit, sum, apart, o);
        if (!ordinary) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) {             // one at a time: registers
                    const float x[1] = {fmaf(-of_scales[wave][0][i * 32 + r / 4 * 8 + half * 4 + r % 4], unit_q, acc[i][r])};
                    add_apart(x, sum, apart);
                }
        }
        float added = 0;
        v8h w[2][2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const v4f inverse = *(const v4f *)&of_scales[wave][1][i * 32 + k * 8 + half * 4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float x = __builtin_amdgcn_exp2f(acc[i][4 * k + r]);
                    added = fmaf(x, inverse[r], added);
                    w[i][k & 1][(k >> 1) * 4 + r] = (_Float16)x;
                }
            }
        if (ordinary) sum += added;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int j = 0; j < G; ++j) o[j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(halves_of(values[j][i][k]), w[i][k], o[j], 0, 0, 0);
    };
    for (; u < s.total; ++u) {
        if (__builtin_expect(!ordinary_scales(a, s, s.block(u), page, scale), 0)) break;
        step(std::true_type());
    }
    const bool ordinary = u >= s.total;
    for (; u < s.total; ++u) step(std::false_type());
    const float by = ordinary ? 1.0f : joined_apart(32, sum, apart);
    sum += __shfl_xor(sum, 32);
    const float f = bad >> lane & 1 ? __builtin_nanf("") : sum > 0 ? by / sum : 0.0f;
    if (col >= s.cols) return;
    int column = s.col0 + col;
    asm("" : "+v"(column));                  // found anew: no registers for its row and head in the loop
    const int hq = h * a.group + column % a.group;
    const long row = s.start + column / a.group;
    auto store = [&](auto type) __attribute__((always_inline)) {
        constexpr int T = decltype(type)::value;
        typedef typename Element<T>::type E;
        struct alignas(4 * sizeof(E)) Quad {
            E e[4];
        };
#pragma unroll
        for (int j = 0; j < G; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int d = j * 32 + k * 8 + half * 4;
                float x[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    x[r] = o[j][4 * k + r] * f;
                    asm("" : "+v"(x[r]));            // rounded to 32 bits first, wherever the row lies
                }
                if (d + 4 <= kv.dim && a.out_quads) {
                    Quad quad;
#pragma unroll
                    for (int r = 0; r < 4; ++r) quad.e[r] = (E)x[r];
                    *(Quad *)((E *)a.out.data + row * a.out.stride + hq * kv.dim + d) = quad;
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (d + r < kv.dim) store_value<T>(a.out, row, hq * kv.dim + d + r, x[r]);
                }
            }
    };
    if (a.out.type == GALA_F16)
        store(std::integral_constant<int, GALA_F16>());
    else
        store(std::integral_constant<int, GALA_BF16>());
}

}  // namespace

namespace gala {

size_t kv4_attention_workspace(const KvArgs &kv, int heads_q, int window, int sinks) {
    const Cut c = cut_of(kv, heads_q, window, sinks, true);          // the other way needs none
    return c.splits == 1 ? 0 : (size_t)kv.count * kv.heads * c.places() * (kv.dim + 2) * sizeof(float);
}

int launch_kv4_attention(void *stream, const KvArgs &kv, int heads_q, float scale, int window, int sinks, const Values &q,
                         const Values &out, void *workspace) {
    const bool fine = !in_halves(scale, q.type, out.type);
    const Cut c = cut_of(kv, heads_q, window, sinks, fine || !fits_wide(q.type, kv.dim));
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
        constexpr int G = decltype(n32)::value;
        if (c.many) {
            a.ordered = kv.count > 1 && kv.count <= 64 && !window;
            auto many = [&](auto parts) {
                hipLaunchKernelGGL((kv4_attention_many_kernel<G, decltype(parts)::value>), dim3(groups), dim3(64 * kWavesOf), 0, (hipStream_t)stream, a);
            };
            if (q.type != GALA_F16)
                many(std::integral_constant<int, 1>());
            else if constexpr (G <= 6)
                many(std::integral_constant<int, 2>());
            return;
        }
        auto waves = [&](auto w) {
            constexpr int W = decltype(w)::value;
            a.waves = W;
            const unsigned lds = W * c.columns * (32 * G + 1) * sizeof(float);
            if (fine)
                hipLaunchKernelGGL((kv4_attention_kernel<G, 3, true, W>), dim3(groups), dim3(64 * W), lds, (hipStream_t)stream, a);
            else if (q.type == GALA_F16 || out.type == GALA_F16)
                hipLaunchKernelGGL((kv4_attention_kernel<G, 2, false, W>), dim3(groups), dim3(64 * W), lds, (hipStream_t)stream, a);
            else
                hipLaunchKernelGGL((kv4_attention_kernel<G, 1, false, W>), dim3(groups), dim3(64 * W), lds, (hipStream_t)stream, a);
        };
        if constexpr (G <= 4) {
            if (c.waves == 8)
                waves(std::integral_constant<int, 8>());
            else
                waves(std::integral_constant<int, 4>());
        } else {
            waves(std::integral_constant<int, 4>());
        }
        if (c.splits == 1) return;
        const unsigned rows = (unsigned)((long)kv.count * kv.heads * c.tiles * c.columns);
        hipLaunchKernelGGL((kv_attention_join_kernel<(G + 1) / 2>), dim3(rows), dim3(64 * kJoinWaves), 0, (hipStream_t)stream, a);
    };
    switch (kv4_groups(kv.dim)) {
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
