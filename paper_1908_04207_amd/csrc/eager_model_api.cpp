// Host side of the model operators (include/eager_model.h): argument checks, then the launch.
#include "../../include/eager_model.h"
#include "eager_model.h"
#include "eager_model_rules.h"

#include <cmath>

namespace {

bool aligned(const void *p, uintptr_t to) { return p && (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

bool valid_dtype(int dtype) { return dtype == EAGER_F32 || dtype == EAGER_BF16; }

int64_t chunk(int dtype) { return dtype == EAGER_BF16 ? 8 : 4; }     // elements in 16 bytes

// Tokens stay this far from 2^31, so that no tile's end passes it.
constexpr int64_t kMaxTokens = (1ll << 31) - (1ll << 16);
// Tiles are at most 256 rows, so the last byte of one lies within 2^31 bytes of its first (fp32: exactly).
constexpr int64_t kMaxStride = 1ll << 21;
constexpr int64_t kMaxGrid = (1ll << 31) - 1;
// With scales from here to its inverse lse / scale and scale * log2(e) are numbers in fp32.
constexpr float kLeastScale = 0x1p-120f;

bool valid_shape(const eager_packed *s)
{
    return s && s->tokens >= 0 && s->tokens <= kMaxTokens && s->kv_heads >= 1 && s->q_heads >= 1 &&
           s->q_heads <= (1 << 20) && s->q_heads % s->kv_heads == 0 && s->head_dim >= 8 &&
           s->head_dim <= EAGER_MAX_HEAD_DIM && s->head_dim % 8 == 0;
}

bool valid_sequences(const eager_packed *s)
{
    return valid_shape(s) && s->sequences >= 1 && s->sequences <= (1 << 30) && aligned(s->cu_seqlens, 4) &&
           eager::tile_numbers(s->tokens, s->sequences, eager::kAttentionRows) * s->q_heads <= kMaxGrid;
}

// no row or head shares elements with the next one (a broadcast view does)
bool valid_heads(const eager_heads *h, int dtype, const eager_packed *s)
{
    const int64_t c = chunk(dtype);
    return h && (aligned(h->data, 16) || s->tokens == 0) && h->row_stride >= s->head_dim && h->row_stride <= kMaxStride &&
           h->head_stride >= s->head_dim && h->row_stride % c == 0 && h->head_stride % c == 0;
}

eager::Heads heads(const eager_heads *h) { return {h->data, h->row_stride, h->head_stride}; }

int status_of(hipError_t e) { return e == hipSuccess ? EAGER_OK : EAGER_EDEVICE; }

bool fill(eager::NormRopeArgs &a, int dtype, const eager_packed *s, const eager_heads *const x[2],
          const eager_heads *const y[2], const void *wq, const void *wk, const eager_rotation *r, float eps)
{
    if (!valid_dtype(dtype) || !valid_shape(s) || !aligned(wq, 16) || !aligned(wk, 16) || !r ||
        !aligned(r->cos_table, 16) || !aligned(r->sin_table, 16) || !(aligned(r->positions, 4) || s->tokens == 0) || r->table_rows < 1 ||
        !(eps >= 0.0f) || !std::isfinite(eps))
        return false;
    for (int i = 0; i < 2; ++i)
        if (!valid_heads(x[i], dtype, s) || !valid_heads(y[i], dtype, s)) return false;
    a = {};
    for (int i = 0; i < 2; ++i) {
        a.x[i] = heads(x[i]);
        a.y[i] = heads(y[i]);
    }
    a.w[0] = wq;
    a.w[1] = wk;
    a.cos_table = r->cos_table;
    a.sin_table = r->sin_table;
    a.positions = r->positions;
    a.tokens = s->tokens;
    a.table_rows = r->table_rows;
    a.heads[0] = s->q_heads;
    a.heads[1] = s->kv_heads;
    a.dim = s->head_dim;
    a.per_block = eager::norm_rope_tokens_per_block(s->q_heads + s->kv_heads, false);
    a.eps = eps;
    a.inv_dim = 1.0f / static_cast<float>(s->head_dim);
    return true;
}

bool fill(eager::AttentionArgs &a, int dtype, const eager_packed *s, const eager_heads *q, const eager_heads *k,
          const eager_heads *v, const eager_heads *out, const float *lse, float scale)
{
    if (!valid_dtype(dtype) || !valid_sequences(s) || !(scale >= kLeastScale && scale <= 1.0f / kLeastScale) ||
        !(aligned(lse, 4) || s->tokens == 0))
        return false;
    for (const eager_heads *h : {q, k, v, out})
        if (!valid_heads(h, dtype, s)) return false;
    a = {};
    a.q = heads(q);
    a.k = heads(k);
    a.v = heads(v);
    a.out = heads(out);
    a.lse = const_cast<float *>(lse);
    a.cu = s->cu_seqlens;
    a.tokens = s->tokens;
    a.q_heads = s->q_heads;
    a.kv_heads = s->kv_heads;
    a.dim = s->head_dim;
    a.sequences = s->sequences;
    a.scale = scale;
    return true;
}

bool valid_projection(int dtype, const eager_projection *s)
{
    return valid_dtype(dtype) && s && s->rows >= 0 && s->rows <= kMaxTokens && s->width >= 8 && s->width % 8 == 0 &&
           s->width <= kMaxStride && s->vocab >= 1 && s->vocab <= (1 << 30) &&
           (s->vocab / 128 + 1ll) * (s->rows / 64 + 1) <= kMaxGrid && s->rows * (s->width / 8) / 128 < kMaxGrid;
}

bool fill(eager::CrossEntropyArgs &a, int dtype, const eager_projection *s, const void *x, const void *w,
          const int64_t *target, void *workspace, int64_t workspace_bytes)
{
    const int64_t c = chunk(dtype);
    if (!valid_projection(dtype, s) || !aligned(w, 16) || (s->rows && (!aligned(x, 16) || !aligned(target, 8))) || !aligned(workspace, 16) ||
        s->x_stride < s->width || s->x_stride > kMaxStride || s->x_stride % c || s->w_stride < s->width ||
        s->w_stride > kMaxStride || s->w_stride % c)
        return false;
    a = {};
    a.x = x;
    a.w = w;
    a.target = reinterpret_cast<const long long *>(target);
    a.workspace = static_cast<char *>(workspace);
    a.rows = s->rows;
    a.x_stride = s->x_stride;
    a.w_stride = s->w_stride;
    a.width = s->width;
    a.vocab = s->vocab;
    a.workspace_bytes = workspace_bytes;
    return true;
}

}  // namespace

extern "C" {

int eager_qk_norm_rope(int dtype, const eager_packed *shape, const eager_heads *q, const eager_heads *k,
                       const void *wq, const void *wk, const eager_rotation *rotation, float eps,
                       const eager_heads *q_out, const eager_heads *k_out, void *stream)
{
    const eager_heads *const x[2] = {q, k}, *const y[2] = {q_out, k_out};
    eager::NormRopeArgs a;
    if (!fill(a, dtype, shape, x, y, wq, wk, rotation, eps)) return EAGER_EINVAL;
    if (a.tokens == 0) return EAGER_OK;
    return status_of(eager::launch_norm_rope(a, dtype == EAGER_BF16, static_cast<hipStream_t>(stream)));
}

int eager_qk_norm_rope_workspace_bytes(int dtype, const eager_packed *shape, int64_t *bytes)
{
    if (!valid_dtype(dtype) || !valid_shape(shape) || !bytes) return EAGER_EINVAL;
    const int64_t blocks = eager::norm_rope_blocks(shape->tokens, shape->q_heads, shape->kv_heads);
    *bytes = (blocks > 0 ? blocks : 1) * 2 * shape->head_dim * 4;
    return EAGER_OK;
}

int eager_qk_norm_rope_backward(int dtype, const eager_packed *shape, const eager_heads *dq_out,
                                const eager_heads *dk_out, const eager_heads *q, const eager_heads *k,
                                const void *wq, const void *wk, const eager_rotation *rotation, float eps,
                                const eager_heads *dq, const eager_heads *dk, void *dwq, void *dwk,
                                void *workspace, int64_t workspace_bytes, void *stream)
{
    const eager_heads *const x[2] = {q, k}, *const y[2] = {dq_out, dk_out};
    eager::NormRopeArgs a;
    int64_t need = 0;
    if (!fill(a, dtype, shape, x, y, wq, wk, rotation, eps) || !valid_heads(dq, dtype, shape) ||
        !valid_heads(dk, dtype, shape) || !aligned(dwq, 4) || !aligned(dwk, 4) || !aligned(workspace, 16) ||
        eager_qk_norm_rope_workspace_bytes(dtype, shape, &need) != EAGER_OK || workspace_bytes < need)
        return EAGER_EINVAL;
    a.dx[0] = heads(dq);
    a.dx[1] = heads(dk);
    a.dw[0] = dwq;
    a.dw[1] = dwk;
    a.partials = static_cast<float *>(workspace);
    a.per_block = eager::norm_rope_tokens_per_block(a.heads[0] + a.heads[1], true);
    a.blocks = eager::norm_rope_blocks(a.tokens, a.heads[0], a.heads[1]);
    return status_of(eager::launch_norm_rope_backward(a, dtype == EAGER_BF16, static_cast<hipStream_t>(stream)));
}

int eager_attention(int dtype, const eager_packed *shape, const eager_heads *q, const eager_heads *k,
                    const eager_heads *v, float scale, const eager_heads *out, float *lse, void *stream)
{
    eager::AttentionArgs a;
    if (!fill(a, dtype, shape, q, k, v, out, lse, scale)) return EAGER_EINVAL;
    if (a.tokens == 0) return EAGER_OK;
    return status_of(eager::launch_attention(a, dtype == EAGER_BF16, static_cast<hipStream_t>(stream)));
}

int eager_attention_workspace_bytes(int dtype, const eager_packed *shape, int64_t *bytes)
{
    if (!valid_dtype(dtype) || !valid_shape(shape) || shape->sequences < 1 || !bytes) return EAGER_EINVAL;
    *bytes = eager::attention_workspace_bytes(shape->tokens, shape->q_heads, shape->kv_heads, shape->head_dim,
                                              shape->sequences);
    return EAGER_OK;
}

int eager_attention_backward(int dtype, const eager_packed *shape, const eager_heads *q, const eager_heads *k,
                             const eager_heads *v, const eager_heads *out, const float *lse,
                             const eager_heads *dout, float scale, const eager_heads *dq,
                             const eager_heads *dk, const eager_heads *dv, void *workspace,
                             int64_t workspace_bytes, void *stream)
{
    eager::AttentionArgs a;
    if (!fill(a, dtype, shape, q, k, v, out, lse, scale)) return EAGER_EINVAL;
    for (const eager_heads *h : {dout, dq, dk, dv})
        if (!valid_heads(h, dtype, shape)) return EAGER_EINVAL;
    if (a.tokens == 0) return EAGER_OK;
    if (!aligned(workspace, 16) || 
        workspace_bytes < eager::attention_workspace_bytes(a.tokens, a.q_heads, a.kv_heads, a.dim, a.sequences))
        return EAGER_EINVAL;
    a.dout = heads(dout);
    a.dq = heads(dq);
    a.dk = heads(dk);
    a.dv = heads(dv);
    a.delta = static_cast<float *>(workspace);
    a.start = a.delta + eager::attention_row_bytes(a.tokens, a.q_heads) / 4;
    a.sums = a.start + eager::attention_row_bytes(a.tokens, a.q_heads) / 4;
    a.parts = eager::attention_parts(a.tokens, a.q_heads, a.kv_heads, a.sequences);
    return status_of(eager::launch_attention_backward(a, dtype == EAGER_BF16, static_cast<hipStream_t>(stream)));
}

int eager_cross_entropy_workspace_bytes(int dtype, const eager_projection *shape, int backward, int64_t *bytes)
{
    if (!valid_projection(dtype, shape) || !bytes || (backward != 0 && backward != 1)) return EAGER_EINVAL;
    *bytes = eager::cross_entropy_workspace_bytes(shape->rows, shape->width, shape->vocab, dtype == EAGER_BF16, backward);
    return EAGER_OK;
}

int eager_cross_entropy(int dtype, const eager_projection *shape, const void *x, const void *w,
                        const int64_t *target, float *loss, float *lse, void *workspace,
                        int64_t workspace_bytes, void *stream)
{
    eager::CrossEntropyArgs a;
    int64_t need = 0;
    if (!fill(a, dtype, shape, x, w, target, workspace, workspace_bytes) ||
        (shape->rows && (!aligned(loss, 4) || !aligned(lse, 4))) ||
        eager_cross_entropy_workspace_bytes(dtype, shape, 0, &need) != EAGER_OK || workspace_bytes < need)
        return EAGER_EINVAL;
    if (a.rows == 0) return EAGER_OK;
    a.loss = loss;
    a.lse = lse;
    return status_of(eager::launch_cross_entropy(a, dtype == EAGER_BF16, static_cast<hipStream_t>(stream)));
}

int eager_cross_entropy_backward(int dtype, const eager_projection *shape, const void *x, const void *w,
                                 const int64_t *target, const float *lse, const float *dloss, void *dx,
                                 void *dw, void *workspace, int64_t workspace_bytes, void *stream)
{
    eager::CrossEntropyArgs a;
    int64_t need = 0;
    if (!fill(a, dtype, shape, x, w, target, workspace, workspace_bytes) ||
        (shape->rows && (!aligned(lse, 4) || !aligned(dloss, 4))) ||
        (!dx && !dw && shape->rows) || (dx && !aligned(dx, 16)) || (dw && !aligned(dw, 16)) ||
        eager_cross_entropy_workspace_bytes(dtype, shape, 1, &need) != EAGER_OK || workspace_bytes < need)
        return EAGER_EINVAL;
    a.lse = const_cast<float *>(lse);
    a.dloss = dloss;
    a.dx = dx;
    a.dw = dw;
    return status_of(eager::launch_cross_entropy_backward(a, dtype == EAGER_BF16, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
