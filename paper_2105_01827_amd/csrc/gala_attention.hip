// Attention of a batch's queries over the paged 8-bit cache.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "gala_decode.h"

using namespace gala;

namespace {

// One wavefront: one query head of one token.  A lane takes a token of a block for the scores, and channels for the sum.
template <int TYPE, int OUT>
__global__ __launch_bounds__(64) void kv_attention_kernel(KvArgs kv, int heads_q, float scale, int window, int sinks, Values q, Values out) {
    __shared__ float qs[kMaxHeadDim], ps[64];
    const int unit = blockIdx.x, hq = unit % heads_q, bi = unit / heads_q, b = bi / kv.max_new, i = bi % kv.max_new;
    const int start = kv.starts[b], n = kv.starts[b + 1] - start, lane = threadIdx.x;
    if (i >= n) return;
    const int at = kv.lens[b] - n + i, h = hq / (heads_q / kv.heads), dim = kv.dim;
    const long row = start + i;
    bool bad = false;
    for (int d = lane; d < kv.dim16 * 16; d += 64) {
        const float x = d < dim ? load_value<TYPE>(q, row, hq * dim + d) : 0.0f;
        bad |= !(fabsf(x) < INFINITY);
        qs[d] = x;
    }
    bad = __any(bad);
    __syncthreads();
    float top = -INFINITY, sum = 0, acc[4] = {0, 0, 0, 0};
    const int end = min(at + 1, kv.max_len);
    for (int block = 0; block * kKvBlock < end; ++block) {
        const int t = block * kKvBlock + lane, last = block * kKvBlock + 63;
        if (window && last <= at - window && block * kKvBlock >= sinks) continue;
        const int page = page_of(kv, b, block);
        if (page < 0) continue;
        const signed char *codes = kv.codes + ((long)page * kv.heads + h) * kv_head_bytes(kv.dim16);
        const float *scales = kv.scales + ((long)page * kv.heads + h) * 2;
        const bool seen = t < end && (!window || t > at - window || t < sinks);
        float dot = 0;
        for (int d = 0; d < kv.dim16 * 16; ++d)
            dot += qs[d] * (float)codes[((lane >> 4) * kv.dim16 + (d >> 4)) * 256 + (lane & 15) * 16 + (d & 15)];
        const float s = seen ? dot * scales[0] * scale : -INFINITY;
        float m = s;
        for (int k = 32; k; k >>= 1) m = fmaxf(m, __shfl_xor(m, k));
        if (m == -INFINITY) continue;
        m = fmaxf(m, top);
        const float was = expf(top - m), p = expf(s - m);
        float all = p;
        for (int k = 32; k; k >>= 1) all += __shfl_xor(all, k);
        sum = sum * was + all;
        top = m;
        __syncthreads();
        ps[lane] = p * scales[1];
        __syncthreads();
        for (int k = 0; k < 4; ++k) {
            const int d = lane + 64 * k;
            if (d >= dim) break;
            float a = 0;
            for (int u = 0; u < 64; ++u)
                a += ps[u] * (float)codes[kKvBlock * 16 * kv.dim16 + (d >> 4) * 1024 + ((u & 15) >> 2) * 256 + (d & 15) * 16 + (u >> 4) * 4 + (u & 3)];
            acc[k] = acc[k] * was + a;
        }
    }
    for (int k = 0; k < 4; ++k) {
        const int d = lane + 64 * k;
        if (d < dim) store_value<OUT>(out, row, hq * dim + d, bad ? __builtin_nanf("") : sum > 0 ? acc[k] / sum : 0.0f);
    }
}

}  // namespace

namespace gala {

size_t kv_attention_workspace(const KvArgs &, int, int, int) { return 0; }

int launch_kv_attention(void *stream, const KvArgs &kv, int heads_q, float scale, int window, int sinks, const Values &q,
                        const Values &out, void *) {
    by_type(q.type, [&](auto type) {
        by_type(out.type, [&](auto to) {
            hipLaunchKernelGGL((kv_attention_kernel<decltype(type)::value, decltype(to)::value>), dim3(kv.count * kv.max_new * heads_q),
                               dim3(64), 0, (hipStream_t)stream, kv, heads_q, scale, window, sinks, q, out);
        });
    });
    return hipGetLastError() != hipSuccess;
}

}  // namespace gala
