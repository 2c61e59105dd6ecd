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

bool fill(eager::CrossEntropyArgs &a, int dtype, const eager_projection *s, const void *x, const void *w, void *workspace,
          int64_t workspace_bytes)
{
    const int64_t c = chunk(dtype);
    if (!valid_projection(dtype, s) || !aligned(w, 16) || (s->rows && !aligned(x, 16)) || !aligned(workspace, 16) ||
        s->x_stride < s->width || s->x_stride > kMaxStride || s->x_stride % c || s->w_stride < s->width ||
        s->w_stride > kMaxStride || s->w_stride % c)
        return false;
    a = {};
    a.x = x;
    a.w = w;
    a.workspace = static_cast<char *>(workspace);
    a.rows = s->rows;
    a.x_stride = s->x_stride;
    a.w_stride = s->w_stride;
    a.width = s->width;
    a.vocab = s->vocab;
    a.workspace_bytes = workspace_bytes;
    return true;
}

// An output in the place of an input is laid out like it.
bool same_or_apart(const eager_heads *x, const eager_heads *y, int64_t tokens, int32_t count)
{
    return x->data != y->data || ((tokens < 2 || x->row_stride == y->row_stride) && (count < 2 || x->head_stride == y->head_stride));
}
bool same_or_apart(const eager_rows *x, const eager_rows *y, int64_t rows)
{
    return !x || !y || x->data != y->data || rows < 2 || x->stride == y->stride;
}

// rows of one array: on 16 bytes, none shares elements with the next one
bool valid_rows(const eager_rows *r, int dtype, int64_t rows, int32_t width)
{
    return r && (aligned(r->data, 16) || rows == 0) && r->stride >= width && r->stride <= kMaxStride && r->stride % chunk(dtype) == 0;
}

eager::Rows rows_of(const eager_rows *r) { return r ? eager::Rows{r->data, r->stride} : eager::Rows{}; }

bool valid_norm(int dtype, int64_t rows, int32_t width)
{
    return valid_dtype(dtype) && rows >= 0 && rows <= kMaxTokens && width >= 8 && width <= EAGER_MAX_NORM_WIDTH && width % 8 == 0;
}
static_assert(eager::kNormWidth == EAGER_MAX_NORM_WIDTH, "the lanes of a workgroup hold the widest row");

// forward and backward (sign -1) alike
int rotate(int dtype, const eager_packed *s, const eager_heads *q, const eager_heads *k, const eager_rotation *r, int32_t part,
           int layout, const eager_heads *q_out, const eager_heads *k_out, float sign, void *stream)
{
    const eager_heads *const x[2] = {q, k}, *const y[2] = {q_out, k_out};
    if (!valid_dtype(dtype) || !valid_shape(s) || !r || !aligned(r->cos_table, 16) || !aligned(r->sin_table, 16) ||
        !(aligned(r->positions, 4) || s->tokens == 0) || r->table_rows < 1 || part < 8 || part > s->head_dim || part % 8 ||
        (layout != EAGER_ROTARY_HALVES && layout != EAGER_ROTARY_INTERLEAVED))
        return EAGER_EINVAL;
    for (int i = 0; i < 2; ++i)
        if (!valid_heads(x[i], dtype, s) || !valid_heads(y[i], dtype, s)) return EAGER_EINVAL;
    if (s->tokens == 0) return EAGER_OK;
    for (int i = 0; i < 2; ++i)
        if (!same_or_apart(x[i], y[i], s->tokens, i ? s->kv_heads : s->q_heads)) return EAGER_EINVAL;
    eager::RotaryArgs a = {};
    a.heads[0] = s->q_heads;
    a.heads[1] = s->kv_heads;
    for (int i = 0; i < 2; ++i) {
        a.x[i] = heads(x[i]);
        a.y[i] = heads(y[i]);
        a.groups[i] = (a.heads[i] + eager::kTurnedHeads - 1) / eager::kTurnedHeads;
        a.moved[i] = x[i]->data == y[i]->data ? part : s->head_dim;
    }
    a.cos_table = r->cos_table;
    a.sin_table = r->sin_table;
    a.positions = r->positions;
    a.tokens = s->tokens;
    a.table_rows = r->table_rows;
    a.half = part / 2;
    a.sign = sign;
    return status_of(eager::launch_rotary(a, dtype == EAGER_BF16, layout == EAGER_ROTARY_INTERLEAVED, static_cast<hipStream_t>(stream)));
}

// The products' grids hold more rows than the lists' kernels, whose workgroups of 1024 threads take 16 each.
constexpr int64_t kMaxTaught = 1 << 25;
constexpr float kLeastTemperature = 0x1p-20f;

bool taught(eager::CrossEntropyArgs &a, const eager_teacher *t, int64_t rows)
{
    if (!t || rows > kMaxTaught || t->entries < 1 || t->entries > EAGER_MAX_ENTRIES ||
        !(t->temperature >= kLeastTemperature && t->temperature <= 1.0f / kLeastTemperature) ||
        (rows && (!aligned(t->index, 8) || !aligned(t->logits, 4))))
        return false;
    a.teacher.index = reinterpret_cast<const long long *>(t->index);
    a.teacher.logits = t->logits;
    a.teacher.entries = t->entries;
    a.teacher.temperature = t->temperature;
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
    if (!fill(a, dtype, shape, x, w, workspace, workspace_bytes) ||
        (shape->rows && (!aligned(target, 8) || !aligned(loss, 4) || !aligned(lse, 4))) ||
        eager_cross_entropy_workspace_bytes(dtype, shape, 0, &need) != EAGER_OK || workspace_bytes < need)
        return EAGER_EINVAL;
    if (a.rows == 0) return EAGER_OK;
    a.target = reinterpret_cast<const long long *>(target);
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
    if (!fill(a, dtype, shape, x, w, workspace, workspace_bytes) ||
        (shape->rows && (!aligned(target, 8) || !aligned(lse, 4) || !aligned(dloss, 4))) ||
        (!dx && !dw && shape->rows) || (dx && !aligned(dx, 16)) || (dw && !aligned(dw, 16)) ||
        eager_cross_entropy_workspace_bytes(dtype, shape, 1, &need) != EAGER_OK || workspace_bytes < need)
        return EAGER_EINVAL;
    a.target = reinterpret_cast<const long long *>(target);
    a.lse = const_cast<float *>(lse);
    a.dloss = dloss;
    a.dx = dx;
    a.dw = dw;
    return status_of(eager::launch_cross_entropy_backward(a, dtype == EAGER_BF16, static_cast<hipStream_t>(stream)));
}

int eager_distillation_workspace_bytes(int dtype, const eager_projection *shape, int32_t entries, int backward, int64_t *bytes)
{
    if (!valid_projection(dtype, shape) || shape->rows > kMaxTaught || entries < 1 || entries > EAGER_MAX_ENTRIES || !bytes ||
        (backward != 0 && backward != 1))
        return EAGER_EINVAL;
    *bytes = eager::distillation_workspace_bytes(shape->rows, shape->width, shape->vocab, entries, dtype == EAGER_BF16, backward);
    return EAGER_OK;
}

int eager_distillation(int dtype, const eager_projection *shape, const void *x, const void *w, const eager_teacher *teacher,
                       float *loss, float *lse, float *picked, void *workspace, int64_t workspace_bytes, void *stream)
{
    eager::CrossEntropyArgs a;
    int64_t need = 0;
    if (!fill(a, dtype, shape, x, w, workspace, workspace_bytes) || !taught(a, teacher, shape->rows) ||
        (shape->rows && (!aligned(loss, 4) || !aligned(lse, 4) || !aligned(picked, 4))) ||
        eager_distillation_workspace_bytes(dtype, shape, teacher->entries, 0, &need) != EAGER_OK || workspace_bytes < need)
        return EAGER_EINVAL;
    if (a.rows == 0) return EAGER_OK;
    a.loss = loss;
    a.lse = lse;
    a.teacher.picked = picked;
    return status_of(eager::launch_cross_entropy(a, dtype == EAGER_BF16, static_cast<hipStream_t>(stream)));
}

int eager_distillation_backward(int dtype, const eager_projection *shape, const void *x, const void *w,
                                const eager_teacher *teacher, const float *lse, const float *picked, const float *dloss, void *dx,
                                void *dw, void *workspace, int64_t workspace_bytes, void *stream)
{
    eager::CrossEntropyArgs a;
    int64_t need = 0;
    if (!fill(a, dtype, shape, x, w, workspace, workspace_bytes) || !taught(a, teacher, shape->rows) ||
        (shape->rows && (!aligned(lse, 4) || !aligned(picked, 4) || !aligned(dloss, 4))) || (!dx && !dw && shape->rows) ||
        (dx && !aligned(dx, 16)) || (dw && !aligned(dw, 16)) ||
        eager_distillation_workspace_bytes(dtype, shape, teacher->entries, 1, &need) != EAGER_OK || workspace_bytes < need)
        return EAGER_EINVAL;
    a.lse = const_cast<float *>(lse);
    a.teacher.picked = const_cast<float *>(picked);
    a.dloss = dloss;
    a.dx = dx;
    a.dw = dw;
    return status_of(eager::launch_cross_entropy_backward(a, dtype == EAGER_BF16, static_cast<hipStream_t>(stream)));
}

int eager_layer_norm(int dtype, int64_t rows, int32_t width, const eager_rows *x, const eager_rows *residual, const void *w,
                     const void *b, float eps, const eager_rows *sum, const eager_rows *y, float *stats, void *stream)
{
    if (!valid_norm(dtype, rows, width) || !valid_rows(x, dtype, rows, width) || !valid_rows(y, dtype, rows, width) ||
        !residual != !sum || (residual && (!valid_rows(residual, dtype, rows, width) || !valid_rows(sum, dtype, rows, width))) ||
        !aligned(w, 16) || (b && !aligned(b, 16)) || !(eps >= 0.0f) || !std::isfinite(eps) || !(aligned(stats, 4) || rows == 0) ||
        (rows && sum && sum->data == y->data))
        return EAGER_EINVAL;
    for (const eager_rows *to : {sum, y})
        if (!same_or_apart(x, to, rows) || !same_or_apart(residual, to, rows)) return EAGER_EINVAL;
    if (rows == 0) return EAGER_OK;
    eager::LayerNormArgs a = {};
    a.x = rows_of(x);
    a.residual = rows_of(residual);
    a.sum = rows_of(sum);
    a.y = rows_of(y);
    a.w = w;
    a.b = b;
    a.stats = stats;
    a.rows = rows;
    a.width = width;
    a.eps = eps;
    a.inv_width = 1.0f / static_cast<float>(width);
    return status_of(eager::launch_layer_norm(a, dtype == EAGER_BF16, static_cast<hipStream_t>(stream)));
}

int eager_layer_norm_workspace_bytes(int dtype, int64_t rows, int32_t width, int64_t *bytes)
{
    if (!valid_norm(dtype, rows, width) || !bytes) return EAGER_EINVAL;
    *bytes = eager::layer_norm_workspace_bytes(rows, width);
    return EAGER_OK;
}

int eager_layer_norm_backward(int dtype, int64_t rows, int32_t width, const eager_rows *dy, const eager_rows *ds,
                              const eager_rows *s, const void *w, const float *stats, const eager_rows *dx, void *dw, void *db,
                              void *workspace, int64_t workspace_bytes, void *stream)
{
    const int64_t need = valid_norm(dtype, rows, width) ? eager::layer_norm_workspace_bytes(rows, width) : 0;
    if (!valid_norm(dtype, rows, width) || !valid_rows(dy, dtype, rows, width) || (ds && !valid_rows(ds, dtype, rows, width)) ||
        !valid_rows(s, dtype, rows, width) || !valid_rows(dx, dtype, rows, width) || !aligned(w, 16) ||
        !(aligned(stats, 4) || rows == 0) || (dw && !aligned(dw, 4)) || (db && !aligned(db, 4)) || (need && !aligned(workspace, 16)) ||
        workspace_bytes < need || !same_or_apart(dy, dx, rows) || !same_or_apart(ds, dx, rows))
        return EAGER_EINVAL;
    eager::LayerNormArgs a = {};
    a.x = rows_of(s);
    a.residual = rows_of(ds);
    a.sum = rows_of(dx);
    a.y = rows_of(dy);
    a.w = w;
    a.dw = dw;
    a.db = db;
    a.stats = const_cast<float *>(stats);
    a.partials = static_cast<float *>(workspace);
    a.rows = rows;
    a.width = width;
    a.blocks = eager::layer_norm_blocks(rows, width);
    a.inv_width = 1.0f / static_cast<float>(width);
    return status_of(eager::launch_layer_norm_backward(a, dtype == EAGER_BF16, static_cast<hipStream_t>(stream)));
}

int eager_rotary_table(const eager_angles *t, float *cos_table, float *sin_table, void *stream)
{
    if (!t || t->positions < 0 || t->positions > kMaxTokens || t->part < 8 || t->part > EAGER_MAX_HEAD_DIM || t->part % 8 ||
        t->scaling < EAGER_ANGLES_PLAIN || t->scaling > EAGER_ANGLES_PARTS || !(t->base >= 1.0) || !std::isfinite(t->base) ||
        !std::isfinite(t->magnitude) || (t->positions && (!aligned(cos_table, 16) || !aligned(sin_table, 16))))
        return EAGER_EINVAL;
    if (t->scaling != EAGER_ANGLES_PLAIN && (!(t->factor >= 1.0) || !std::isfinite(t->factor))) return EAGER_EINVAL;
    if (t->scaling == EAGER_ANGLES_PARTS && (!(t->original > 0.0) || !std::isfinite(t->original) || !(t->low >= 0.0) ||
                                             !(t->high > t->low) || !std::isfinite(t->high)))
        return EAGER_EINVAL;
    if (t->positions == 0) return EAGER_OK;
    constexpr double kPi = 3.14159265358979323846;
    eager::TableArgs a = {};
    const double n = t->part, stretched = t->scaling == EAGER_ANGLES_BASE ? t->base * std::pow(t->factor, n / (n - 2)) : t->base;
    for (int i = 0; i < t->part / 2; ++i) {
        double f = std::pow(stretched, -2.0 * i / n);
        if (t->scaling == EAGER_ANGLES_LINEAR) f /= t->factor;
        if (t->scaling == EAGER_ANGLES_PARTS) {
            const double turns = t->original * f / (2 * kPi);
            const double keep = std::fmin(std::fmax((turns - t->low) / (t->high - t->low), 0.0), 1.0);
            f *= keep + (1 - keep) / t->factor;
        }
        a.quarters[i] = f * (2 / kPi);
    }
    a.magnitude = t->magnitude;
    a.cos_table = cos_table;
    a.sin_table = sin_table;
    a.positions = t->positions;
    a.half = t->part / 2;
    return status_of(eager::launch_rotary_table(a, static_cast<hipStream_t>(stream)));
}

int eager_rotary(int dtype, const eager_packed *shape, const eager_heads *q, const eager_heads *k, const eager_rotation *rotation,
                 int32_t part, int layout, const eager_heads *q_out, const eager_heads *k_out, void *stream)
{
    return rotate(dtype, shape, q, k, rotation, part, layout, q_out, k_out, 1.0f, stream);
}

int eager_rotary_backward(int dtype, const eager_packed *shape, const eager_heads *dq_out, const eager_heads *dk_out,
                          const eager_rotation *rotation, int32_t part, int layout, const eager_heads *dq, const eager_heads *dk,
                          void *stream)
{
    return rotate(dtype, shape, dq_out, dk_out, rotation, part, layout, dq, dk, -1.0f, stream);
}

}  // extern "C"
