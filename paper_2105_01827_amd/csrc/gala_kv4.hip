// Keys and values of new tokens into the paged 4-bit cache, positions rotated in on the way, and rows of the cache back as
// floats.
// A code is x / s to the nearest of eight magnitudes.  Of a key s is the smallest power of two with max|x| <= 7 s over 32 channels
// (6 s with what rounds to it), so that its codes times s are exact in bfloat16; of a value s = max|x| / 6 over the head in 16 bits,
// a factor of the token's weight.  Either depends on one token alone: nothing that is there is read or rounded again.
#include "gala_rows.h"

using namespace gala;

namespace {

constexpr int kThreads = 256;
constexpr float kLeastScale = 0x1p-100f;         // of a value

// Offsets within a head's part of a page: the word of a key's eight codes from channel d on (a multiple of 8), and the word of a
// value's eight codes of channel d that token t is among.
__device__ __forceinline__ int key_word(int t, int d, int groups) { return ((t >> 4) * groups + (d >> 5)) * 256 + (t & 15) * 16 + ((d & 31) >> 1); }
__device__ __forceinline__ int value_word(int t, int d, int groups) {
    return 1024 * groups + (d >> 5) * 1024 + ((t & 15) >> 2) * 256 + (d & 15) * 16 + ((d & 31) >> 4) * 8 + (t >> 5) * 4;
}
// which of that word's codes: tokens 4p .. 4p+3 of 32, then those 16 further on
__device__ __forceinline__ int slot_of(int t) { return (t & 31) / 16 * 4 + (t & 3); }
__device__ __forceinline__ int token_of(int half, int part, int slot) { return 32 * half + 16 * (slot >> 2) + 4 * part + (slot & 3); }

// Eight words of eight codes each: word c gets code c of all of them.
__device__ __forceinline__ void transpose_codes(u32 (&w)[8]) {
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        const u32 x = w[s], y = w[s + 4];
        w[s] = __builtin_amdgcn_perm(y, x, 0x05040100), w[s + 4] = __builtin_amdgcn_perm(y, x, 0x07060302);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int s = (k & 1) + (k >> 1) * 4;
        const u32 x = w[s], y = w[s + 2];
        w[s] = __builtin_amdgcn_perm(y, x, 0x06020400), w[s + 2] = __builtin_amdgcn_perm(y, x, 0x07030501);
    }
#pragma unroll
    for (int s = 0; s < 8; s += 2) {
        const u32 x = w[s], y = w[s + 1];
        w[s] = (x & 0x0f0f0f0fu) | (y & 0x0f0f0f0fu) << 4, w[s + 1] = (x >> 4 & 0x0f0f0f0fu) | (y & 0xf0f0f0f0u);
    }
}

// eight codes, the nearest to x / scale for a power of two (the conversion's own rounding: ties to the even code, 6 beyond 6)
__device__ __forceinline__ u32 codes_of(const float (&x)[8], float scale) {
    u32 w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
}
// ... and what they stand for; the product with the scale is the caller's
__device__ __forceinline__ void floats_of(u32 w, float (&x)[8]) {
    typedef float v2f __attribute__((ext_vector_type(2)));
    const v2f a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1);
    const v2f c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3);
    x[0] = a[0], x[1] = a[1], x[2] = b[0], x[3] = b[1], x[4] = c[0], x[5] = c[1], x[6] = d[0], x[7] = d[1];
}

// one member of a pair; products and the sum rounded one by one
__device__ __forceinline__ float turned_by(float cos, float sin, float own, float other) {
#pragma clang fp contract(off)
    return cos * own + sin * other;
}
// A piece of eight channels of a row's head, as floats, 0 behind the head's end; of keys with the position rotated in (NaN where the
// table does not have it).  `pieces`: rows are read in pieces, and pairs lie in them.
template <int TYPE>
__device__ __forceinline__ void load_rotated(const Values &x, bool pieces, const RopeArgs &rope, long row, int t, int h, int d, int dim, float (&v)[8]) {
    const bool has = !rope.table || (t >= 0 && t < rope.positions);
    const float *table = rope.table && has ? rope.table + (long)t * rope.half * 2 : nullptr;
    if (pieces) {
        // loads without branches between them, so that those of several pieces are under way together
        const bool turned = rope.table && d < 2 * rope.half, second = !rope.interleaved && d >= rope.half;
        const int own = d < dim ? d : 0, partner = !turned || rope.interleaved ? own : second ? d - rope.half : d + rope.half;
        load_piece<TYPE>(x, row, h * dim + own, v);
        if (rope.table) {
            const long at = has ? t : 0;
            const int pair = !turned ? 0 : rope.interleaved ? d / 2 : second ? d - rope.half : d;
            float angles[16], other[8];
            const float4 *from = (const float4 *)(rope.table + (at * rope.half + pair) * 2);
#pragma unroll
            for (int k = 0; k < 2; ++k) *(float4 *)(angles + 4 * k) = from[k];
            if (!rope.interleaved) {
#pragma unroll
                for (int k = 2; k < 4; ++k) *(float4 *)(angles + 4 * k) = from[k];
                load_piece<TYPE>(x, row, h * dim + partner, other);
            }
            if (turned) {
                if (rope.interleaved) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) turn_pair(angles[2 * k], angles[2 * k + 1], v[2 * k], v[2 * k + 1]);
                } else {
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] = turned_by(angles[2 * k], second ? angles[2 * k + 1] : -angles[2 * k + 1], v[k], other[k]);
                }
            }
        }
        if (d >= dim) {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = 0;
            return;
        }
    } else {
        auto row_at = [&](int c) { return load_value<TYPE>(x, row, h * dim + c); };
        RopeArgs r = rope;
        r.table = table;
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = d + k < dim ? rotated(r, table, d + k, row_at) : 0.0f;
    }
    if (!has) {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = __builtin_nanf("");
    }
}
// the largest finite magnitude of eight numbers; NaN among them becomes 0.  `infinite`: infinities may be among them.
__device__ __forceinline__ float clean(float (&v)[8], bool &infinite) {
    u32 bits[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) bits[k] = __float_as_uint(v[k]) & 0x7fffffffu;
    u32 most = max(max(max(bits[0], bits[1]), max(bits[2], bits[3])), max(max(bits[4], bits[5]), max(bits[6], bits[7])));
    infinite = __any(most >= 0x7f800000u);
    if (infinite) {
        most = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (bits[k] > 0x7f800000u) v[k] = 0;
            if (bits[k] < 0x7f800000u) most = max(most, bits[k]);
        }
    }
    return __uint_as_float(most);
}

// The new tokens of one touched block of one sequence: [lo, hi) of the sequence, which lie in `page`.
struct Block {
    int start, first, at, lo, hi, page;      // `at`: the block's first token; row of token t: start + t - first
};
__device__ __forceinline__ Block block_of(const KvArgs &kv, int b, int j) {
    Block o;
    o.start = kv.starts[b];
    const int n = kv.starts[b + 1] - o.start;
    o.first = kv.lens[b] - n;
    const int block = max(o.first, 0) / kKvBlock + j;
    o.at = block * kKvBlock;
    o.lo = max(o.first, o.at), o.hi = min(o.first + min(n, kv.max_new), o.at + kKvBlock);
    o.page = o.lo < o.hi ? page_of(kv, b, block) : -1;
    return o;
}

// One workgroup: the keys of one head in one touched block.  Four lanes have a token's 32 channels: its largest comes from two
// exchanges within four lanes, its codes are a word a lane, 16 consecutive bytes a group.  Bound by the wait for rows (half of a wavefront's
// time); 5609 tokens of four sequences, 4 heads of 128 f16 channels with 16 heads of queries, 61 MB, take 13.0 us where the last-level cache has them, 16.7 from HBM.
template <int TYPE, int THREADS>
__device__ void append_keys(const KvArgs &kv, const RopeArgs &rope, const Values &x, bool pieces, int h, const Block &o) {
    const int groups = kv4_groups(kv.dim), count = o.hi - o.lo;
    char *data = (char *)kv.codes + ((size_t)o.page * kv.heads + h) * kv4_head_bytes(groups);
    const Divisor of(4 * groups);
    // one piece at a time: two under way take registers from other wavefronts (4000 tokens of 24 heads of 80: 34.6 us against 30.7)
    for (int e = threadIdx.x; e < count * 4 * groups; e += THREADS) {
        const int i = of(e), d = (e - i * 4 * groups) * 8, t = o.lo + i - o.at;
        float v[8];
        load_rotated<TYPE>(x, pieces, rope, o.start + (o.lo + i - o.first), o.lo + i, h, d, kv.dim, v);
        bool infinite;
        float most = clean(v, infinite);
        most = fmaxf(most, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(most), 0xb1, 0xf, 0xf, true)));        // of the four lanes
        most = fmaxf(most, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(most), 0x4e, 0xf, 0xf, true)));
        // most = f * 2^e with 1 <= f < 2: at most 7 * 2^(e-2) if f <= 7/4
        const u32 bits = __float_as_uint(most);
        const int exponent = min(max((int)(bits >> 23) - 127 - 2 + ((bits & 0x7fffffu) > 0x600000u), kLeastExponent), kMostExponent);
        *(u32 *)(data + key_word(t, d, groups)) = codes_of(v, __uint_as_float((u32)(exponent + 127) << 23));
        if ((e & 3) == 0) data[kv4_exponents(groups) + (d >> 5) * 64 + (t & 15) * 4 + (t >> 4)] = (char)(exponent + 127);
    }
}

// One workgroup: the values of one head in one touched block.  A token's scale needs its whole row, a word of codes eight tokens of
// a channel: rows stay in registers until their scale is there, their codes wait in LDS, and eight words of a channel piece of eight
// tokens each are turned by three steps of exchanges of halves, bytes and nibbles.  A word that old tokens share is read and written
// by the one thread that has it.
template <int TYPE, int THREADS, int MOST>
__device__ void append_values(const KvArgs &kv, const Values &x, bool pieces, int h, const Block &o, u32 (*tile)[33], u32 *largest) {
    // items a thread may have: MOST groups of 32 channels, THREADS / 4 tokens
    constexpr int kItems = MOST;
    const int groups = kv4_groups(kv.dim), count = o.hi - o.lo, tid = threadIdx.x, t_lo = o.lo - o.at, t_hi = o.hi - o.at;
    char *data = (char *)kv.codes + ((size_t)o.page * kv.heads + h) * kv4_head_bytes(groups);
    const Divisor of(4 * groups);
    const RopeArgs none{nullptr, 0, 0, 0};
    if (tid < kKvBlock) largest[tid] = 0;
    __syncthreads();
    float v[kItems][8];
    bool infinite[kItems];
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        const int e = tid + k * THREADS, i = of(e), d = (e - i * 4 * groups) * 8;
        infinite[k] = false;
        if (i < count) {
            load_rotated<TYPE>(x, pieces, none, o.start + (o.lo + i - o.first), o.lo + i, h, d, kv.dim, v[k]);
            atomicMax(&largest[t_lo + i], __float_as_uint(clean(v[k], infinite[k])));
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        const int e = tid + k * THREADS, i = of(e), d = (e - i * 4 * groups) * 8, t = t_lo + i;
        if (i < count) {
            const __bf16 rounded_scale = (__bf16)(__uint_as_float(largest[t]) * (1.0f / 6.0f));
            float scale = (float)rounded_scale;
            if (scale < kLeastScale) scale = 0;
            const float inverse = scale > 0 ? 1.0f / scale : 0.0f;
            float q[8];
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                // the quotient rounded once: the remainder of a first one is exact
                const float first = v[k][c] * inverse, rest = fmaf(-first, scale, v[k][c]);
                q[c] = copysignf(fmaf(rest, inverse, first), v[k][c]);
            }
            if (infinite[k]) {
#pragma unroll
                for (int c = 0; c < 8; ++c) q[c] = fabsf(v[k][c]) < INFINITY ? q[c] : v[k][c];
            }
            tile[t][d >> 3] = scale > 0 ? codes_of(q, 1.0f) : 0;
            if (d == 0) *(__bf16 *)(data + kv4_scales(groups) + ((t & 15) >> 2) * 32 + (t >> 4) * 8 + (t & 3) * 2) = (__bf16)scale;
        }
    }
    __syncthreads();
    // eight channels of eight tokens at a time: 16 bytes of a channel by neighbouring lanes
    for (int e = tid; e < groups * 32; e += THREADS) {
        const int half = e & 1, piece = (e >> 5) * 4 + (e >> 1 & 1) * 2 + (e >> 4 & 1), part = e >> 2 & 3;
        u32 mask = 0, w[8];
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            const int t = token_of(half, part, s);
            const bool is_new = t >= t_lo && t < t_hi;
            mask |= is_new ? 0xfu << 4 * s : 0;
            w[s] = is_new ? tile[t][piece] : 0;
        }
        if (!mask) continue;
        transpose_codes(w);
        u32 *to = (u32 *)(data + value_word(token_of(half, part, 0), piece * 8, groups));
#pragma unroll
        for (int c = 0; c < 8; ++c) to[4 * c] = mask == ~0u ? w[c] : (to[4 * c] & ~mask) | w[c];
    }
}

// Workgroups of a launch: one for the keys and one for the values of each head in each touched block, then those with some
// tokens' queries each, `rows` of a sequence.
struct Shares {
    Order order;
    int blocks, groups, rows;
    Turns turns;
};

// Six wavefronts a SIMD where heads are narrow: registers that the compiler takes beyond that cost more than they save (the
// prompts above from HBM 16.7 us against 17.7, eight 17.1; from the cache 13.0, 13.0 and 12.6).
template <int TYPE, int OUT, int THREADS, int MOST>
__global__ __launch_bounds__(THREADS, MOST == 4 ? 6 : 1) void kv4_append_kernel(KvArgs kv, RopeArgs rope, int heads_q, Values q, Values q_out, Values k, Values v,
                                                             Shares shares, bool pieces) {
    __shared__ u32 tile[kKvBlock][33], largest[kKvBlock];
    if ((int)blockIdx.x < shares.groups) {
        const int2 unit = shares.order.unit_of(blockIdx.x);
        if (unit.x >= shares.order.blocks) return;
        const int which = unit.y & 1, h = unit.y >> 1, b = unit.x / shares.blocks;
        const Block o = block_of(kv, b, unit.x - b * shares.blocks);
        if (o.page < 0) return;
        if (which)
            append_values<TYPE, THREADS, MOST>(kv, v, pieces, h, o, tile, largest);
        else
            append_keys<TYPE, THREADS>(kv, rope, k, pieces, h, o);
    } else {
        const int all = blockIdx.x - shares.groups, u = all / shares.turns.parts, part = all - u * shares.turns.parts;
        const int b = u / shares.rows, i0 = (u - b * shares.rows) * shares.turns.rows;
        if (pieces) {
            const int start = kv.starts[b], n = kv.starts[b + 1] - start, first = kv.lens[b] - n, most = min(n, kv.max_new);
            turn_heads<TYPE, OUT, THREADS>(shares.turns, part, q, q_out, [&](int r) { return i0 + r < most ? (long)start + i0 + r : -1; },
                                           [&](int r, bool two, bool turned, int d, float(&angle)[16]) __attribute__((always_inline)) {
                const int t = first + i0 + r;
                const bool has = !rope.table || (t >= 0 && t < rope.positions);
                if (rope.table && has && turned) {
                    const float4 *from = (const float4 *)(rope.table + ((long)t * rope.half + (two ? d : d / 2)) * 2);
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (k < 2 || two) {
                            const float4 x = from[k];
                            angle[4 * k] = x.x, angle[4 * k + 1] = x.y, angle[4 * k + 2] = x.z, angle[4 * k + 3] = x.w;
                        }
                }
                return has;
            });
        } else {
            for (int i = i0; i < min(i0 + shares.turns.rows, kv.max_new); ++i) rotate_row<TYPE, OUT, THREADS>(kv, rope, q, q_out, heads_q, b * kv.max_new + i);
        }
    }
}

// One workgroup: the keys or the values of one head in one block of one sequence.  A code times its scale is rounded once, to the output's
// type.  Values: eight words, turned as they were on their way in, are eight channels of eight tokens.  5810 tokens of 4 heads of
// 128 f16 channels, 15 MB, take 6.2 us, 7.2 from HBM; blocks of 64 sequences 7.9 us; four pieces under way gain nothing.
template <int OUT>
__global__ __launch_bounds__(kThreads) void kv4_export_kernel(KvArgs kv, Values k_out, Values v_out, int blocks, Order order, bool pieces) {
    const int2 unit = order.unit_of(blockIdx.x);
    if (unit.x >= order.blocks) return;
    const int which = unit.y & 1, h = unit.y >> 1, b = unit.x / blocks, j = unit.x - b * blocks;
    const int start = kv.starts[b], n = kv.starts[b + 1] - start, first = kv.lens[b] - n;
    // tokens at negative positions are in blocks of their own numbers, down from -1
    const int block = (first >= 0 ? first / kKvBlock : -((63 - first) / kKvBlock)) + j, at = block * kKvBlock;
    const int lo = max(first, at) - at, hi = min(first + min(n, kv.max_new), at + kKvBlock) - at;
    if (lo >= hi) return;
    const int page = page_of(kv, b, block), groups = kv4_groups(kv.dim);
    const Values &out = which ? v_out : k_out;
    const char *data = (const char *)kv.codes + ((size_t)max(page, 0) * kv.heads + h) * kv4_head_bytes(groups);
    auto put = [&](int t, int d, u32 word, float scale) {
        float x[8];
        floats_of(word, x);
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] *= scale;
        const long row = start + (at + t - first);
        if (pieces) {
            store_piece<OUT>(out, row, h * kv.dim + d, x);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (d + k < kv.dim) store_value<OUT>(out, row, h * kv.dim + d + k, x[k]);
        }
    };
    if (!which || page < 0) {
        const Divisor of(4 * groups);
        for (int e = threadIdx.x; e < (hi - lo) * 4 * groups; e += kThreads) {
            const int i = of(e), d = (e - i * 4 * groups) * 8, t = lo + i;
            if (d >= kv.dim) continue;
            if (page < 0) {
                put(t, d, 0, 1.0f);
                continue;
            }
            const u32 exponent = ((const unsigned char *)data)[kv4_exponents(groups) + (d >> 5) * 64 + (t & 15) * 4 + (t >> 4)];
            put(t, d, *(const u32 *)(data + key_word(t, d, groups)), __uint_as_float(exponent << 23));
        }
        return;
    }
    for (int e = threadIdx.x; e < groups * 32; e += kThreads) {
        const int piece = (e >> 5) * 4 + (e & 3), half = e >> 2 & 1, part = e >> 3 & 3, d = piece * 8;
        if (d >= kv.dim) continue;
        u32 w[8];
        const u32 *from = (const u32 *)(data + value_word(token_of(half, part, 0), d, groups));
#pragma unroll
        for (int c = 0; c < 8; ++c) w[c] = from[4 * c];
        transpose_codes(w);
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            const int t = token_of(half, part, s);
            if (t >= lo && t < hi)
                put(t, d, w[s], (float)*(const __bf16 *)(data + kv4_scales(groups) + part * 32 + (t >> 4) * 8 + (t & 3) * 2));
        }
    }
}

}  // namespace

namespace gala {

int launch_kv4_append(void *stream, const KvArgs &kv, const RopeArgs &rope, int heads_q, const Values &q, const Values &q_out,
                      const Values &k, const Values &v) {
    // the most blocks that max_new tokens in a row can touch
    const int blocks = (kv.max_new + kKvBlock - 2) / kKvBlock + 1;
    const bool pieces = in_pieces(q, kv.dim) && in_pieces(q_out, kv.dim) && in_pieces(k, kv.dim) && in_pieces(v, kv.dim) &&
                        (!rope.table || ((uintptr_t)rope.table % 16 == 0 && rope.half % (rope.interleaved ? 4 : 8) == 0)) &&
                        (long)heads_q * kv.dim / 8 < 65536;
    by_type(k.data ? k.type : q.type, [&](auto type) {
        by_type(q_out.type, [&](auto out) {
            constexpr int T = decltype(type)::value, O = decltype(out)::value;
            if constexpr (O != GALA_RESIDUE) {
                auto launch = [&](auto threads, auto most) {
                    constexpr int N = decltype(threads)::value, M = decltype(most)::value;
                    Shares s{order_of(k.data ? kv.count * blocks : 0, kv.heads, kv.dim, k), blocks, 0, 0,
                             turns_of((long)kv.count * kv.max_new, std::max(1, heads_q), kv.dim, rope.half, rope.interleaved, N)};
                    s.turns.rows = pieces ? std::min(s.turns.rows, kv.max_new) : 1;
                    if (!pieces) s.turns.parts = 1;
                    s.groups = s.order.groups();
                    s.rows = (kv.max_new + s.turns.rows - 1) / s.turns.rows;
                    hipLaunchKernelGGL((kv4_append_kernel<T, O, N, M>), dim3(s.groups + (heads_q ? kv.count * s.rows * s.turns.parts : 0)), dim3(N), 0,
                                       (hipStream_t)stream, kv, rope, heads_q, q, q_out, k, v, s, pieces);
                };
                // a wavefront a workgroup where a sequence has few tokens (what four would hold, they would wait for); a thread's items by the
                // head's size, so that registers of eight pieces are kept for heads that have them
                const bool few = kv.max_new <= 16, narrow = kv.dim <= 128;
                if (few && narrow) launch(std::integral_constant<int, 64>(), std::integral_constant<int, 4>());
                if (few && !narrow) launch(std::integral_constant<int, 64>(), std::integral_constant<int, 8>());
                if (!few && narrow) launch(std::integral_constant<int, 256>(), std::integral_constant<int, 4>());
                if (!few && !narrow) launch(std::integral_constant<int, 256>(), std::integral_constant<int, 8>());
            }
        });
    });
    return hipGetLastError() != hipSuccess;
}

int launch_kv4_export(void *stream, const KvArgs &kv, const Values &k_out, const Values &v_out) {
    const int blocks = (kv.max_new + kKvBlock - 2) / kKvBlock + 1;
    const Order order = order_of(kv.count * blocks, kv.heads, kv.dim, k_out);
    const bool pieces = in_pieces(k_out, kv.dim) && in_pieces(v_out, kv.dim);
    by_type(k_out.type, [&](auto type) {
        hipLaunchKernelGGL((kv4_export_kernel<decltype(type)::value>), dim3(order.groups()), dim3(kThreads), 0, (hipStream_t)stream, kv, k_out, v_out,
                           blocks, order, pieces);
    });
    return hipGetLastError() != hipSuccess;
}

}  // namespace gala
