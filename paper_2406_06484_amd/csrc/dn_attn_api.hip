// C ABI of the attention operators (declared in include/deltanet.h): validation, workspace sizes, dispatch.  Host code only.
#include "../../include/deltanet.h"
#include "dn_attn_host.hpp"

#include <math.h>
#include <string.h>

namespace {

using namespace dn;

constexpr int kMostTokens = 1 << 30; // 32-bit positions and rows, and some tiles or strides past the last

bool misaligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }
int elem_bytes(int dtype) { return dtype == DN_BF16 ? 2 : 4; }

// rows of H heads of d elements, `stride` elements apart
int check_rows(int64_t stride, int H, int d, int es) {
    if (stride < (int64_t)H * d || stride > ((int64_t)1 << 31)) return DN_ERR_SHAPE;
    return stride * es % 16 == 0 ? DN_OK : DN_ERR_ALIGN;
}

int check_heads(int T, int Hq, int Hkv, int dtype) {
    if (T < 0 || T > kMostTokens || Hq <= 0 || Hkv <= 0 || Hq > 8192 || Hkv > Hq || Hq % Hkv) return DN_ERR_SHAPE;
    if ((long long)T * Hq >= (1ll << 31)) return DN_ERR_SHAPE; // 32-bit indices of rows and heads
    return dtype == DN_F32 || dtype == DN_BF16 ? DN_OK : DN_ERR_UNSUPPORTED;
}

int check_rope(const dn_rope *r, int d, const float *cos_sin) {
    if (!r) return DN_ERR_NULL;
    if (r->rot < 0 || r->rot > d || !(r->eps >= 0.f) || isinf(r->eps)) return DN_ERR_SHAPE;
    if (r->rot % 16) return DN_ERR_UNSUPPORTED;
    if (r->rot && !cos_sin) return DN_ERR_NULL;
    return r->rot && r->max_pos <= 0 ? DN_ERR_SHAPE : DN_OK;
}

int check_qk(const dn_qk_shape *s) {
    if (!s) return DN_ERR_NULL;
    if (int rc = check_heads(s->T, s->Hq, s->Hkv, s->dtype)) return rc;
    if (s->d != 32 && s->d != 64 && s->d != 128 && s->d != 256) return DN_ERR_UNSUPPORTED;
    if (int rc = check_rows(s->q_stride, s->Hq, s->d, elem_bytes(s->dtype))) return rc;
    return check_rows(s->k_stride, s->Hkv, s->d, elem_bytes(s->dtype));
}

int check_paged(const dn_paged_shape *s) {
    if (!s) return DN_ERR_NULL;
    if (int rc = check_heads(s->T, s->Hq, s->Hkv, s->dtype)) return rc;
    const bool d_ok = s->dtype == DN_F32 ? s->d == 32 || s->d == 64 || s->d == 128 : s->d == 64 || s->d == 128 || s->d == 256;
    if (!d_ok) return DN_ERR_UNSUPPORTED;
    if (s->cache_dtype != s->dtype && !(s->cache_dtype == DN_FP8 && s->dtype == DN_BF16)) return DN_ERR_UNSUPPORTED;
    const int ps = s->page_size;
    if (ps != 16 && ps != 32 && ps != 64 && ps != 128 && ps != 256) return DN_ERR_UNSUPPORTED;
    if (s->num_seqs < 0 || s->num_seqs > 65535 || s->num_pages < 0 || s->max_pages < 0 || s->max_q < 0 || s->max_kv < 0) return DN_ERR_SHAPE;
    if (s->max_q > s->T || (long long)s->max_kv > (long long)s->max_pages * ps) return DN_ERR_SHAPE;
    if (s->max_kv > kMostTokens) return DN_ERR_SHAPE;
    if (s->num_pages == 0 && s->max_kv > 0) return DN_ERR_SHAPE;
    if ((long long)s->Hkv * ps * s->d * elem_bytes(s->dtype) >= (1ll << 30)) return DN_ERR_SHAPE; // a page lies within a buffer descriptor's range
    return DN_OK;
}

int check_cache(const dn_paged_shape *s, const dn_paged_cache *c) {
    if (!c) return DN_ERR_NULL;
    if (s->num_seqs && (!s->cu_q || !s->kv_len)) return DN_ERR_NULL;
    if (s->max_kv && s->num_seqs) {
        if (!s->page_table || !c->k_pages || !c->v_pages) return DN_ERR_NULL;
        if (s->cache_dtype == DN_FP8 && (!c->k_scale || !c->v_scale)) return DN_ERR_NULL;
    }
    const void *al[] = {c->k_pages, c->v_pages, c->k_scale, c->v_scale, s->cu_q, s->kv_len, s->page_table};
    for (const void *p : al) if (misaligned(p)) return DN_ERR_ALIGN;
    return DN_OK;
}

PagedArgs paged_args(const dn_paged_shape *s, const dn_paged_cache *c) {
    PagedArgs a;
    a.kp = c->k_pages; a.vp = c->v_pages; a.ks = c->k_scale; a.vs = c->v_scale;
    a.cu = s->cu_q; a.kv_len = s->kv_len; a.table = s->page_table;
    a.N = s->num_seqs;
    a.page_shift = __builtin_ctz((unsigned)s->page_size);
    a.num_pages = s->num_pages; a.max_pages = s->max_pages; a.max_kv = s->max_kv;
    return a;
}

RowArgs row_args(int T, int Hq, int Hkv) {
    RowArgs a;
    memset(&a, 0, sizeof(a));
    a.T = T; a.Hq = Hq; a.Hkv = Hkv;
    return a;
}
void set_rope(RowArgs *a, const dn_rope *r, const void *qw, const void *kw, const float *cs) {
    a->qw = qw; a->kw = kw; a->cs = cs;
    a->rot = r->rot; a->interleaved = r->interleaved != 0; a->max_pos = r->max_pos; a->eps = r->eps;
}

int done(int rc) { return rc == 0 ? DN_OK : DN_ERR_LAUNCH; }

int append(const dn_paged_shape *s, const dn_rope *rope, const void *q, const void *k, const void *v, const void *q_weight,
           const void *k_weight, const float *cos_sin, void *q_out, const dn_paged_cache *cache, bool norm, void *hip_stream) {
    if (int rc = check_paged(s)) return rc;
    const int es = elem_bytes(s->dtype);
    if (norm) {
        if (int rc = check_rope(rope, s->d, cos_sin)) return rc;
        if (int rc = check_rows(s->q_stride, s->Hq, s->d, es)) return rc;
    }
    if (int rc = check_rows(s->k_stride, s->Hkv, s->d, es)) return rc;
    if (int rc = check_rows(s->v_stride, s->Hkv, s->d, es)) return rc;
    if (s->T && (!k || !v || (norm && (!q || !q_out)))) return DN_ERR_NULL;
    if (int rc = check_cache(s, cache)) return rc;
    const void *al[] = {q, k, v, q_weight, k_weight, cos_sin, q_out};
    for (const void *p : al) if (misaligned(p)) return DN_ERR_ALIGN;
    RowArgs a = row_args(s->T, s->Hq, s->Hkv);
    a.q = q; a.k = k; a.v = v; a.q_out = q_out;
    a.q_stride = s->q_stride; a.k_stride = s->k_stride; a.v_stride = s->v_stride;
    if (norm) set_rope(&a, rope, q_weight, k_weight, cos_sin);
    return done(run_paged_append(s->dtype, s->d, s->cache_dtype == DN_FP8, norm, a, paged_args(s, cache), static_cast<hipStream_t>(hip_stream)));
}

AttnArgs attn_args(const dn_paged_shape *s, const dn_paged_cache *c, int window) {
    AttnArgs a;
    a.r = row_args(s->T, s->Hq, s->Hkv);
    a.r.q_stride = s->q_stride;
    a.c = paged_args(s, c);
    a.scale = 0.f;
    a.window = window >= s->max_kv ? 0 : window; // (a window as long as any context hides nothing)
    a.max_q = s->max_q; a.splits = 1;
    a.zero_front = a.zero_rest = 1;
    a.workspace = nullptr;
    return a;
}

} // namespace

extern "C" {

int deltanet_qk_norm_rope_fwd(const dn_qk_shape *shape, const dn_rope *rope, const void *q, const void *k, const void *q_weight,
                              const void *k_weight, const float *cos_sin, const int32_t *positions, void *q_out, void *k_out,
                              void *hip_stream) {
    if (int rc = check_qk(shape)) return rc;
    if (int rc = check_rope(rope, shape->d, cos_sin)) return rc;
    if (!positions && shape->seq_len <= 0) return DN_ERR_SHAPE;
    if (shape->T && (!q || !k || !q_out || !k_out)) return DN_ERR_NULL;
    const void *al[] = {q, k, q_weight, k_weight, cos_sin, positions, q_out, k_out};
    for (const void *p : al) if (misaligned(p)) return DN_ERR_ALIGN;
    RowArgs a = row_args(shape->T, shape->Hq, shape->Hkv);
    a.q = q; a.k = k; a.q_out = q_out; a.k_out = k_out;
    a.q_stride = shape->q_stride; a.k_stride = shape->k_stride;
    a.positions = positions; a.seq_len = shape->seq_len;
    set_rope(&a, rope, q_weight, k_weight, cos_sin);
    return done(run_norm_rope_fwd(shape->dtype, shape->d, a, static_cast<hipStream_t>(hip_stream)));
}

int deltanet_qk_norm_rope_workspace_bytes(const dn_qk_shape *shape, size_t *out_bytes) {
    if (!out_bytes) return DN_ERR_NULL;
    if (int rc = check_qk(shape)) return rc;
    *out_bytes = (size_t)norm_rope_bwd_blocks(shape->T) * 2 * shape->d * sizeof(float);
    return DN_OK;
}

int deltanet_qk_norm_rope_bwd(const dn_qk_shape *shape, const dn_rope *rope, const void *q, const void *k, const void *dq_out,
                              const void *dk_out, const void *q_weight, const void *k_weight, const float *cos_sin,
                              const int32_t *positions, void *dq, void *dk, float *dq_weight, float *dk_weight, void *workspace,
                              size_t workspace_bytes, void *hip_stream) {
    size_t need = 0;
    if (int rc = deltanet_qk_norm_rope_workspace_bytes(shape, &need)) return rc;
    if (int rc = check_rope(rope, shape->d, cos_sin)) return rc;
    if (!positions && shape->seq_len <= 0) return DN_ERR_SHAPE;
    if (shape->T && (!q || !k || !dq_out || !dk_out || !dq || !dk)) return DN_ERR_NULL;
    const void *al[] = {q, k, dq_out, dk_out, q_weight, k_weight, cos_sin, positions, dq, dk, dq_weight, dk_weight, workspace};
    for (const void *p : al) if (misaligned(p)) return DN_ERR_ALIGN;
    const bool sums = dq_weight || dk_weight;
    if (sums && need && (!workspace || workspace_bytes < need)) return DN_ERR_WORKSPACE;
    RowArgs a = row_args(shape->T, shape->Hq, shape->Hkv);
    a.q = q; a.k = k; a.dq_out = dq_out; a.dk_out = dk_out; a.q_out = dq; a.k_out = dk;
    a.q_stride = shape->q_stride; a.k_stride = shape->k_stride;
    a.positions = positions; a.seq_len = shape->seq_len;
    a.partial = sums ? static_cast<float *>(workspace) : nullptr;
    a.dqw = dq_weight; a.dkw = dk_weight;
    set_rope(&a, rope, q_weight, k_weight, cos_sin);
    return done(run_norm_rope_bwd(shape->dtype, shape->d, a, static_cast<hipStream_t>(hip_stream)));
}

int deltanet_paged_append(const dn_paged_shape *shape, const void *k, const void *v, const dn_paged_cache *cache, void *hip_stream) {
    return append(shape, nullptr, nullptr, k, v, nullptr, nullptr, nullptr, nullptr, cache, false, hip_stream);
}

int deltanet_paged_norm_rope_append(const dn_paged_shape *shape, const dn_rope *rope, const void *q, const void *k, const void *v,
                                    const void *q_weight, const void *k_weight, const float *cos_sin, void *q_out,
                                    const dn_paged_cache *cache, void *hip_stream) {
    return append(shape, rope, q, k, v, q_weight, k_weight, cos_sin, q_out, cache, true, hip_stream);
}

int deltanet_paged_read(const dn_paged_shape *shape, const dn_paged_cache *cache, const int32_t *cu_out, int32_t T_out, void *k_out,
                        void *v_out, void *hip_stream) {
    if (int rc = check_paged(shape)) return rc;
    if (T_out < 0 || T_out > kMostTokens || (long long)T_out * shape->Hkv >= (1ll << 31)) return DN_ERR_SHAPE;
    if (int rc = check_cache(shape, cache)) return rc;
    if (T_out && (!k_out || !v_out)) return DN_ERR_NULL;
    if (shape->num_seqs && !cu_out) return DN_ERR_NULL;
    const void *al[] = {cu_out, k_out, v_out};
    for (const void *p : al) if (misaligned(p)) return DN_ERR_ALIGN;
    RowArgs a = row_args(T_out, shape->Hq, shape->Hkv);
    a.k_out = k_out; a.v_out = v_out;
    PagedArgs c = paged_args(shape, cache);
    c.cu = cu_out;
    return done(run_paged_read(shape->dtype, shape->d, shape->cache_dtype == DN_FP8, a, c, static_cast<hipStream_t>(hip_stream)));
}

int deltanet_paged_attn_workspace_bytes(const dn_paged_shape *shape, int32_t window, size_t *out_bytes) {
    if (!out_bytes) return DN_ERR_NULL;
    if (int rc = check_paged(shape)) return rc;
    if (window < 0) return DN_ERR_SHAPE;
    if (shape->dtype == DN_F32 && (long long)shape->max_q * shape->Hq >= (1ll << 26)) return DN_ERR_SHAPE; // a sequence's tiles of 16 rows are one launch's
    const dn_paged_cache none = {nullptr, nullptr, nullptr, nullptr};
    *out_bytes = paged_attn_workspace(shape->dtype, shape->d, attn_args(shape, &none, window));
    return DN_OK;
}

int deltanet_paged_attn_fwd(const dn_paged_shape *shape, const void *q, const dn_paged_cache *cache, float scale, int32_t window,
                            void *o, void *workspace, size_t workspace_bytes, void *hip_stream) {
    size_t need = 0;
    if (int rc = deltanet_paged_attn_workspace_bytes(shape, window, &need)) return rc;
    if (!(scale > 0.f) || isinf(scale)) return DN_ERR_SHAPE;
    if (int rc = check_rows(shape->q_stride, shape->Hq, shape->d, elem_bytes(shape->dtype))) return rc;
    if (shape->T && (!q || !o)) return DN_ERR_NULL;
    if (int rc = check_cache(shape, cache)) return rc;
    const void *al[] = {q, o, workspace};
    for (const void *p : al) if (misaligned(p)) return DN_ERR_ALIGN;
    if (need && (!workspace || workspace_bytes < need)) return DN_ERR_WORKSPACE;
    AttnArgs a = attn_args(shape, cache, window);
    a.r.q = q; a.r.q_out = o;
    a.scale = scale;
    a.workspace = workspace;
    return done(run_paged_attn(shape->dtype, shape->d, shape->cache_dtype == DN_FP8, a, static_cast<hipStream_t>(hip_stream)));
}

} // extern "C"
