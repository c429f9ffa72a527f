// A language model's steps between two linear layers: what their kernels share, and their launchers.
#pragma once
#include <cstddef>

#include "gala_internal.h"

namespace gala {

constexpr int kKvBlock = GALA_KV_BLOCK;
constexpr int kMaxHeadDim = 256;

// Values of a call, as kernels take them.
struct Values {
    char *data;
    long stride;             // elements from one row to the next
    float unit;
    u32 p;                   // residues: the plaintext modulus
    int type;
};
// The cache and the sequences of a call, all checked by the host.
struct KvArgs {
    signed char *codes;
    float *scales;
    const int *starts, *lens, *table;
    int heads, dim, dim16;   // dim16: head_dim / 16, rounded up
    int pages, count, max_new, max_len, table_stride;
};
struct RopeArgs {
    const float *table;      // nullptr: nothing is rotated
    int positions, half, interleaved;
};

GALA_HD size_t kv_head_bytes(int dim16) { return (size_t)2 * kKvBlock * 16 * dim16; }

int launch_kv_append(void *stream, const KvArgs &kv, const RopeArgs &rope, int heads_q, const Values &q, const Values &q_out,
                     const Values &k, const Values &v);
int launch_kv_export(void *stream, const KvArgs &kv, const Values &k_out, const Values &v_out);
size_t kv_attention_workspace(const KvArgs &kv, int heads_q, int window, int sinks);
int launch_kv_attention(void *stream, const KvArgs &kv, int heads_q, float scale, int window, int sinks, const Values &q,
                        const Values &out, void *workspace);
size_t sample_workspace(int rows, int vocab);
int launch_sample(void *stream, const Values &logits, int rows, int vocab, const gala_sampling &how, int *tokens,
                  void *workspace);

#if defined(__HIPCC__)
// Where a page number is kept, or -1 for a token that the call has no page for.
__device__ __forceinline__ int page_of(const KvArgs &kv, int b, int block) {
    if (block < 0 || block >= kv.table_stride) return -1;
    const int page = kv.table[(long)b * kv.table_stride + block];
    return (u32)page < (u32)kv.pages ? page : -1;
}

template <int TYPE>
struct Element;
template <>
struct Element<GALA_F32> { typedef float type; };
template <>
struct Element<GALA_F16> { typedef _Float16 type; };
template <>
struct Element<GALA_BF16> { typedef __bf16 type; };
template <>
struct Element<GALA_RESIDUE> { typedef u64 type; };

// A value in 32 bits.  Of a residue: its representative nearest to zero (rounded to 24 bits where p is larger) times
// the unit.
template <int TYPE>
__device__ __forceinline__ float to_float(typename Element<TYPE>::type x, float unit, u32 p) {
    if constexpr (TYPE == GALA_RESIDUE)
        return (float)(long)(x > (p >> 1) ? x - p : x) * unit;
    else
        return (float)x;
}
template <int TYPE>
__device__ __forceinline__ float load_value(const Values &v, long row, int column) {
    typedef typename Element<TYPE>::type E;
    return to_float<TYPE>(((const E *)v.data)[row * v.stride + column], v.unit, v.p);
}
template <int TYPE>
__device__ __forceinline__ typename Element<TYPE>::type from_float(float x, float unit, u32 p) {
    if constexpr (TYPE == GALA_RESIDUE) {
        const long most = (long)(p >> 1);
        const float t = rintf(x / unit);
        long r = t != t ? 0 : t >= (float)most ? most : t <= -(float)most ? -most : (long)t;
        return (u64)(r < 0 ? r + (long)p : r);
    } else {
        return (typename Element<TYPE>::type)x;
    }
}
template <int TYPE>
__device__ __forceinline__ void store_value(const Values &v, long row, int column, float x) {
    typedef typename Element<TYPE>::type E;
    ((E *)v.data)[row * v.stride + column] = from_float<TYPE>(x, v.unit, v.p);
}
// f with the type as a constant
template <class F>
__host__ __device__ inline void by_type(int type, F f) {
    switch (type) {
        case GALA_F32: f(std::integral_constant<int, GALA_F32>()); break;
        case GALA_F16: f(std::integral_constant<int, GALA_F16>()); break;
        case GALA_BF16: f(std::integral_constant<int, GALA_BF16>()); break;
        default: f(std::integral_constant<int, GALA_RESIDUE>()); break;
    }
}
#endif

}  // namespace gala
