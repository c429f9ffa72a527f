// Entry points of a language model's steps between two linear layers: argument checks and rope tables.  No allocation
// happens here, and nothing waits.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "gala_decode.h"

using namespace gala;

namespace {

constexpr int kFarthest = 1 << 30;      // no sequence is longer: distances beyond it are cut to it
constexpr int kMostTokens = (1 << 24) - 1;      // of a vocabulary: that many weights of 2^40 add up in 64 bits
constexpr double kTwoPi = 6.283185307179586476925286766559;

size_t type_size(int type) { return type == GALA_F32 ? 4 : type == GALA_RESIDUE ? 8 : 2; }

// `row`: numbers of a row; an output's rows must not overlap
bool values_ok(const gala_values *v, int64_t row, bool output) {
    if (!v || !v->data || v->type < GALA_F32 || v->type > GALA_RESIDUE || v->stride < (output ? row : 0)) return false;
    if ((uintptr_t)v->data % type_size(v->type)) return false;
    return v->type != GALA_RESIDUE || (v->unit > 0 && std::isfinite(v->unit));
}
Values values(const gala_ctx *c, const gala_values *v) {
    return v ? Values{(char *)v->data, (long)v->stride, v->unit, (u32)c->p, v->type} : Values{nullptr, 0, 1, 1, GALA_F32};
}
bool cache_ok(const gala_kv_cache *k) {
    if (!k || k->heads < 1 || k->head_dim < 1 || k->head_dim > kMaxHeadDim || k->pages < 0) return false;
    if (k->pages && (!k->codes || !k->scales)) return false;
    return (uintptr_t)k->codes % 16 == 0 && (uintptr_t)k->scales % 4 == 0;
}
bool batch_ok(const gala_kv_batch *b) {
    if (!b || b->count < 0 || b->max_new < 0 || b->max_len < 0 || b->table_stride < 0) return false;
    if (b->count && (!b->starts || !b->lens || (b->table_stride && !b->table))) return false;
    // positions and tokens fit 32 bits with room for a block
    return b->max_new <= kFarthest && b->max_len <= kFarthest && b->table_stride <= (1 << 24);
}
KvArgs kv_args(const gala_kv_cache *k, const gala_kv_batch *b) {
    KvArgs a{};
    a.codes = (signed char *)k->codes;
    a.scales = k->scales;
    a.starts = b->starts, a.lens = b->lens, a.table = b->table;
    a.heads = k->heads, a.dim = k->head_dim, a.dim16 = (k->head_dim + 15) / 16;
    a.pages = k->pages, a.count = b->count, a.max_new = b->max_new, a.max_len = b->max_len, a.table_stride = b->table_stride;
    return a;
}
// what a launch may have in workgroups
bool fits_grid(int64_t groups) { return groups <= 0x7fffffff; }
bool attention_ok(const gala_kv_cache *cache, const gala_kv_batch *batch, int heads_q, int window, int sinks) {
    if (!cache_ok(cache) || !batch_ok(batch) || heads_q < 1 || heads_q % cache->heads || window < 0 || sinks < 0) return false;
    return heads_q <= (1 << 20) && fits_grid((int64_t)batch->count * batch->max_new) &&
           fits_grid((int64_t)batch->count * batch->max_new * heads_q);
}

}  // namespace

extern "C" size_t gala_kv_cache_bytes(int pages, int heads, int head_dim) {
    if (pages < 0 || heads < 1 || head_dim < 1 || head_dim > kMaxHeadDim) return 0;
    return (size_t)pages * heads * kv_head_bytes((head_dim + 15) / 16);
}

extern "C" int gala_rope_table(int positions, int rot_dim, double base, int scaling, double factor, double original,
                               double low, double high, float *table) {
    if (positions < 0 || rot_dim < 2 || rot_dim % 2 || rot_dim > kMaxHeadDim || !(base > 0) || !std::isfinite(base) || !table)
        return GALA_EARG;
    if (scaling < GALA_ROPE_PLAIN || scaling > GALA_ROPE_RAMP) return GALA_EARG;
    if (scaling != GALA_ROPE_PLAIN && !(factor > 0 && std::isfinite(factor))) return GALA_EARG;
    if (scaling == GALA_ROPE_RAMP && !(original > 0 && std::isfinite(original) && low < high)) return GALA_EARG;
    const int half = rot_dim / 2;
    for (int i = 0; i < half; ++i) {
        double f = std::pow(base, -2.0 * i / rot_dim);
        if (scaling == GALA_ROPE_LINEAR) f /= factor;
        if (scaling == GALA_ROPE_RAMP) {
            const double kept = std::fmin(1, std::fmax(0, (original * f / kTwoPi - low) / (high - low)));
            f = f * kept + f / factor * (1 - kept);
        }
        for (int t = 0; t < positions; ++t) {
            table[((size_t)t * half + i) * 2] = (float)std::cos(t * f);
            table[((size_t)t * half + i) * 2 + 1] = (float)std::sin(t * f);
        }
    }
    return GALA_OK;
}

extern "C" int gala_kv_append(const gala_ctx *c, void *stream, const gala_kv_cache *cache, const gala_kv_batch *batch,
                              const gala_rope *rope, int heads_q, const gala_values *q, const gala_values *q_out,
                              const gala_values *k, const gala_values *v) {
    if (!c || !cache_ok(cache) || !batch_ok(batch) || heads_q < 0) return GALA_EARG;
    if (!q != !q_out || !q != !heads_q || !k != !v) return GALA_EARG;
    const int dim = cache->head_dim;
    if (q && (!values_ok(q, (int64_t)heads_q * dim, false) || !values_ok(q_out, (int64_t)heads_q * dim, true) ||
              q_out->type == GALA_RESIDUE))
        return GALA_EARG;
    if (q && q_out->data == q->data && (q_out->type != q->type || q_out->stride != q->stride)) return GALA_EARG;
    if (k && (!values_ok(k, (int64_t)cache->heads * dim, false) || !values_ok(v, (int64_t)cache->heads * dim, false) ||
              k->type != v->type))
        return GALA_EARG;
    if (q && k && q->type != k->type) return GALA_EARG;
    if (rope && (!rope->table || rope->positions < 1 || rope->rot_dim < 2 || rope->rot_dim % 2 || rope->rot_dim > dim ||
                 (uintptr_t)rope->table % 8))
        return GALA_EARG;
    const int64_t blocks = (batch->max_new + 62) / 64 + 1;
    if (heads_q > (1 << 20) || !fits_grid((int64_t)batch->count * batch->max_new) ||
        !fits_grid(((int64_t)batch->count * blocks + 7) * cache->heads * 2 + (int64_t)batch->count * batch->max_new))
        return GALA_EARG;
    if (!c->has_device) return GALA_EHIP;
    if (!batch->count || !batch->max_new || (!q && !k)) return GALA_OK;
    const RopeArgs r{rope ? rope->table : nullptr, rope ? rope->positions : 0, rope ? rope->rot_dim / 2 : 0,
                     rope ? rope->interleaved != 0 : 0};
    return launch_kv_append(stream, kv_args(cache, batch), r, heads_q, values(c, q), values(c, q_out), values(c, k),
                            values(c, v)) ? GALA_EHIP : GALA_OK;
}

extern "C" int gala_kv_export(const gala_ctx *c, void *stream, const gala_kv_cache *cache, const gala_kv_batch *batch,
                              const gala_values *k_out, const gala_values *v_out) {
    if (!c || !cache_ok(cache) || !batch_ok(batch)) return GALA_EARG;
    const int64_t row = (int64_t)cache->heads * cache->head_dim;
    if (!values_ok(k_out, row, true) || !values_ok(v_out, row, true) || k_out->type != v_out->type) return GALA_EARG;
    if (!fits_grid(((int64_t)batch->count * ((batch->max_new + 62) / 64 + 1) + 7) * cache->heads * 2)) return GALA_EARG;
    if (!c->has_device) return GALA_EHIP;
    if (!batch->count || !batch->max_new) return GALA_OK;
    return launch_kv_export(stream, kv_args(cache, batch), values(c, k_out), values(c, v_out)) ? GALA_EHIP : GALA_OK;
}

extern "C" size_t gala_kv_attention_workspace(const gala_kv_cache *cache, const gala_kv_batch *batch, int heads_q, int window,
                                              int sinks) {
    if (!attention_ok(cache, batch, heads_q, window, sinks)) return 0;
    return kv_attention_workspace(kv_args(cache, batch), heads_q, std::min(window, kFarthest), std::min(sinks, kFarthest));
}

extern "C" int gala_kv_attention(const gala_ctx *c, void *stream, const gala_kv_cache *cache, const gala_kv_batch *batch,
                                 int heads_q, float scale, int window, int sinks, const gala_values *q,
                                 const gala_values *out, void *workspace, size_t workspace_bytes) {
    if (!c || !attention_ok(cache, batch, heads_q, window, sinks) || !std::isfinite(scale)) return GALA_EARG;
    const int64_t row = (int64_t)heads_q * cache->head_dim;
    if (!values_ok(q, row, false) || !values_ok(out, row, true)) return GALA_EARG;
    if (out->data == q->data && (out->type != q->type || out->stride != q->stride)) return GALA_EARG;
    const KvArgs kv = kv_args(cache, batch);
    window = std::min(window, kFarthest), sinks = std::min(sinks, kFarthest);
    const size_t need = kv_attention_workspace(kv, heads_q, window, sinks);
    if (need && (!workspace || (uintptr_t)workspace % 16)) return GALA_EARG;
    if (workspace_bytes < need) return GALA_ENOMEM;
    if (!c->has_device) return GALA_EHIP;
    if (!batch->count || !batch->max_new) return GALA_OK;
    return launch_kv_attention(stream, kv, heads_q, scale, window, sinks, values(c, q), values(c, out), workspace) ? GALA_EHIP
                                                                                                                   : GALA_OK;
}

extern "C" size_t gala_sample_workspace(int rows, int vocab) {
    return rows < 0 || vocab < 1 || vocab > kMostTokens ? 0 : sample_workspace(rows, vocab);
}

extern "C" int gala_sample(const gala_ctx *c, void *stream, const gala_values *logits, int rows, int vocab,
                           const gala_sampling *how, int32_t *tokens, void *workspace, size_t workspace_bytes) {
    if (!c || rows < 0 || vocab < 1 || vocab > kMostTokens || !values_ok(logits, vocab, false) || !how || !how->u || !tokens) return GALA_EARG;
    const size_t need = sample_workspace(rows, vocab);
    if (need && (!workspace || (uintptr_t)workspace % 16)) return GALA_EARG;
    if (workspace_bytes < need) return GALA_ENOMEM;
    if (!c->has_device) return GALA_EHIP;
    if (!rows) return GALA_OK;
    return launch_sample(stream, values(c, logits), rows, vocab, *how, tokens, workspace) ? GALA_EHIP : GALA_OK;
}
