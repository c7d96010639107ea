// C ABI of the operators around a mixer (declared in include/deltanet.h): validation, workspace sizes, dispatch.  Host code only.
#include "../../include/deltanet.h"
#include "dn_layer_host.hpp"

#include <math.h>
#include <string.h>

namespace {

using namespace dn;

constexpr int kMostRows = 1 << 30, kMostChannels = 1 << 20, kMostWidth = 8192;

bool misaligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }
int elem_bytes(int dtype) { return dtype == DN_BF16 ? 2 : 4; }
int done(int rc) { return rc == 0 ? DN_OK : DN_ERR_LAUNCH; }

int check_stride(int64_t stride, int64_t least, int es) {
    if (stride < least || stride > ((int64_t)1 << 31)) return DN_ERR_SHAPE;
    return stride * es % 16 == 0 ? DN_OK : DN_ERR_ALIGN;
}
template <int N> int check_align(const void *const (&p)[N]) {
    for (const void *q : p) if (misaligned(q)) return DN_ERR_ALIGN;
    return DN_OK;
}

int check_conv(const dn_conv_shape *s, bool bwd) {
    if (!s) return DN_ERR_NULL;
    if (s->B < 0 || s->L < 0 || (long long)s->B * s->L > kMostRows || s->C <= 0 || s->C > kMostChannels) return DN_ERR_SHAPE;
    if (s->dtype != DN_F32 && s->dtype != DN_BF16) return DN_ERR_UNSUPPORTED;
    if (s->W < 2 || s->W > kMostTaps) return DN_ERR_UNSUPPORTED;
    if (s->parts < 1 || s->parts > kMostParts) return DN_ERR_SHAPE;
    const int es = elem_bytes(s->dtype);
    int64_t sum = 0;
    for (int i = 0; i < s->parts; ++i) {
        if (s->width[i] <= 0) return DN_ERR_SHAPE;
        sum += s->width[i];
    }
    if (sum != s->C) return DN_ERR_SHAPE;
    for (int i = 0; i < s->parts; ++i) if (s->width[i] * (int64_t)es % 16) return DN_ERR_ALIGN;
    if (int rc = check_stride(s->x_stride, s->C, es)) return rc;
    if (bwd) if (int rc = check_stride(s->dx_stride, s->C, es)) return rc;
    if (s->cu_seqlens) {
        if (s->B != 1 || s->num_seqs < 0 || s->num_seqs > kMostRows) return DN_ERR_SHAPE;
        if (misaligned(s->cu_seqlens)) return DN_ERR_ALIGN;
        if (const int32_t *c = s->cu_seqlens_host) {
            if (c[0] != 0 || c[s->num_seqs] != s->L) return DN_ERR_CUSEQLENS;
            for (int n = 0; n < s->num_seqs; ++n) if (c[n + 1] < c[n]) return DN_ERR_CUSEQLENS;
        }
    } else if (s->B > kMostRows) return DN_ERR_SHAPE;
    return DN_OK;
}

ConvArgs conv_args(const dn_conv_shape *s) {
    ConvArgs a;
    memset(&a, 0, sizeof(a));
    a.cu = s->cu_seqlens;
    a.N = s->cu_seqlens ? s->num_seqs : s->B;
    a.L = s->L;
    a.T = s->B * s->L;
    a.C = s->C;
    a.W = s->W;
    a.x_stride = s->x_stride;
    a.dx_stride = s->dx_stride;
    for (int i = 0; i < kMostParts; ++i) {
        a.at[i + 1] = a.at[i] + (i < s->parts ? s->width[i] : 0);
        if (i < s->parts && s->silu[i]) a.silu |= 1 << i;
    }
    return a;
}

int check_out_norm(const dn_out_norm_shape *s) {
    if (!s) return DN_ERR_NULL;
    if (s->T < 0 || s->T > kMostRows || s->H <= 0 || (long long)s->T * s->H >= (1ll << 31)) return DN_ERR_SHAPE;
    if (s->dtype != DN_F32 && s->dtype != DN_BF16) return DN_ERR_UNSUPPORTED;
    if (s->d != 32 && s->d != 64 && s->d != 128 && s->d != 256) return DN_ERR_UNSUPPORTED;
    if (!(s->eps >= 0.f) || isinf(s->eps)) return DN_ERR_SHAPE;
    return check_stride(s->o_stride, (int64_t)s->H * s->d, elem_bytes(s->dtype));
}
int check_gate(const dn_out_norm_shape *s, const void *gate, bool bwd) {
    if (!gate) return DN_OK;
    if (s->act != DN_ACT_SILU && s->act != DN_ACT_SIGMOID) return DN_ERR_UNSUPPORTED;
    const int64_t row = (int64_t)s->H * s->d;
    if (int rc = check_stride(s->gate_stride, row, elem_bytes(s->dtype))) return rc;
    return bwd ? check_stride(s->dgate_stride, row, elem_bytes(s->dtype)) : DN_OK;
}
OutNormArgs out_norm_args(const dn_out_norm_shape *s) {
    OutNormArgs a;
    memset(&a, 0, sizeof(a));
    a.T = s->T; a.H = s->H; a.act = s->act; a.eps = s->eps;
    a.o_stride = s->o_stride; a.gate_stride = s->gate_stride; a.dgate_stride = s->dgate_stride;
    // row / H for rows under 2^31: with 2^l >= H, floor(2^(31 + l) / H) + 1 is over 2^(31 + l) / H by at most 2^l / H of a unit
    if (s->H > 1) {
        int l = 1;
        while ((1ll << l) < s->H) ++l;
        a.magic = (unsigned)((1ull << (31 + l)) / (unsigned)s->H + 1);
        a.shift = l - 1;
    }
    return a;
}

int check_block_norm(const dn_block_norm_shape *s) {
    if (!s) return DN_ERR_NULL;
    if (s->T < 0 || s->T > kMostRows || s->D <= 0) return DN_ERR_SHAPE;
    if (s->dtype != DN_F32 && s->dtype != DN_BF16) return DN_ERR_UNSUPPORTED;
    if (s->stream_dtype != DN_F32 && s->stream_dtype != s->dtype) return DN_ERR_UNSUPPORTED;
    if (s->D % 8 || s->D > kMostWidth) return DN_ERR_UNSUPPORTED;
    if (!(s->eps >= 0.f) || isinf(s->eps) || !isfinite(s->scale) || !isfinite(s->residual_scale)) return DN_ERR_SHAPE;
    return DN_OK;
}
BlockNormArgs block_norm_args(const dn_block_norm_shape *s) {
    BlockNormArgs a;
    memset(&a, 0, sizeof(a));
    a.T = s->T; a.D = s->D; a.eps = s->eps; a.scale = s->scale; a.res_scale = s->residual_scale;
    a.x_stride = s->x_stride; a.res_stride = s->residual_stride;
    return a;
}

} // namespace

extern "C" {

int deltanet_short_conv_fwd(const dn_conv_shape *shape, const void *x, const void *weight, const void *bias, const void *initial_state,
                            void *const *y, void *final_state, void *hip_stream) {
    if (int rc = check_conv(shape, false)) return rc;
    ConvArgs a = conv_args(shape);
    if (!weight || !y || (a.T && !x)) return DN_ERR_NULL;
    for (int i = 0; i < shape->parts; ++i) {
        if (a.T && !y[i]) return DN_ERR_NULL;
        if (misaligned(y[i])) return DN_ERR_ALIGN;
        a.y[i] = y[i];
    }
    if (int rc = check_align({x, weight, bias, initial_state, final_state})) return rc;
    a.x = x; a.w = weight; a.b = bias; a.s0 = initial_state; a.sT = final_state;
    return done(run_short_conv_fwd(shape->dtype, a, static_cast<hipStream_t>(hip_stream)));
}

int deltanet_short_conv_workspace_bytes(const dn_conv_shape *shape, size_t *out_bytes) {
    if (!out_bytes) return DN_ERR_NULL;
    if (int rc = check_conv(shape, false)) return rc;
    const int blocks = short_conv_bwd_blocks(shape->dtype, conv_args(shape));
    *out_bytes = blocks > 1 ? (size_t)blocks * shape->C * (shape->W + 1) * sizeof(float) : 0;
    return DN_OK;
}

int deltanet_short_conv_bwd(const dn_conv_shape *shape, const void *x, const void *weight, const void *const *dy, const void *bias,
                            const void *initial_state, const void *dfinal_state, void *dx, float *dweight, float *dbias,
                            void *dinitial_state, void *workspace, size_t workspace_bytes, void *hip_stream) {
    if (int rc = check_conv(shape, true)) return rc;
    ConvArgs a = conv_args(shape);
    if (!weight || !dy || (a.T && (!x || !dx))) return DN_ERR_NULL;
    for (int i = 0; i < shape->parts; ++i) {
        if (a.T && !dy[i]) return DN_ERR_NULL;
        if (misaligned(dy[i])) return DN_ERR_ALIGN;
        a.dy[i] = dy[i];
    }
    if (int rc = check_align({x, weight, bias, initial_state, dfinal_state, dx, dweight, dbias, dinitial_state, workspace})) return rc;
    size_t need = 0;
    if (int rc = deltanet_short_conv_workspace_bytes(shape, &need)) return rc;
    const bool sums = dweight || dbias;
    if (sums && need && (!workspace || workspace_bytes < need)) return DN_ERR_WORKSPACE;
    a.x = x; a.w = weight; a.b = bias; a.s0 = initial_state; a.dsT = dfinal_state;
    a.dx = dx; a.dw = dweight; a.db = dbias; a.ds0 = dinitial_state;
    a.partial = sums ? static_cast<float *>(workspace) : nullptr;
    return done(run_short_conv_bwd(shape->dtype, a, static_cast<hipStream_t>(hip_stream)));
}

int deltanet_out_norm_fwd(const dn_out_norm_shape *shape, const void *o, const void *gate, const void *weight, void *y, void *hip_stream) {
    if (int rc = check_out_norm(shape)) return rc;
    if (int rc = check_gate(shape, gate, false)) return rc;
    if (shape->T && (!o || !y)) return DN_ERR_NULL;
    if (int rc = check_align({o, gate, weight, y})) return rc;
    OutNormArgs a = out_norm_args(shape);
    a.o = o; a.gate = gate; a.w = weight; a.y = y;
    return done(run_out_norm_fwd(shape->dtype, shape->d, a, static_cast<hipStream_t>(hip_stream)));
}

int deltanet_out_norm_workspace_bytes(const dn_out_norm_shape *shape, size_t *out_bytes) {
    if (!out_bytes) return DN_ERR_NULL;
    if (int rc = check_out_norm(shape)) return rc;
    const int blocks = out_norm_bwd_blocks(shape->dtype, shape->d, shape->T, shape->H);
    *out_bytes = blocks > 1 ? (size_t)blocks * shape->d * sizeof(float) : 0;
    return DN_OK;
}

int deltanet_out_norm_bwd(const dn_out_norm_shape *shape, const void *o, const void *dy, const void *gate, const void *weight, void *d_o,
                          void *dgate, float *dweight, void *workspace, size_t workspace_bytes, void *hip_stream) {
    size_t need = 0;
    if (int rc = deltanet_out_norm_workspace_bytes(shape, &need)) return rc;
    if (int rc = check_gate(shape, gate, true)) return rc;
    if (shape->T && (!o || !dy || !d_o || (gate && !dgate))) return DN_ERR_NULL;
    if (int rc = check_align({o, dy, gate, weight, d_o, dgate, dweight, workspace})) return rc;
    if (dweight && need && (!workspace || workspace_bytes < need)) return DN_ERR_WORKSPACE;
    OutNormArgs a = out_norm_args(shape);
    a.o = o; a.gate = gate; a.w = weight; a.dy = dy;
    a.d_o = d_o; a.dgate = dgate; a.dw = dweight;
    a.partial = dweight ? static_cast<float *>(workspace) : nullptr;
    return done(run_out_norm_bwd(shape->dtype, shape->d, a, static_cast<hipStream_t>(hip_stream)));
}

int deltanet_block_norm_fwd(const dn_block_norm_shape *shape, const void *x, const void *residual, const void *weight, const void *gate,
                            void *y, void *h, void *hip_stream) {
    if (int rc = check_block_norm(shape)) return rc;
    if (int rc = check_stride(shape->x_stride, shape->D, elem_bytes(shape->dtype))) return rc;
    if (residual) if (int rc = check_stride(shape->residual_stride, shape->D, elem_bytes(shape->stream_dtype))) return rc;
    if (shape->T && (!x || !y)) return DN_ERR_NULL;
    if (int rc = check_align({x, residual, weight, gate, y, h})) return rc;
    BlockNormArgs a = block_norm_args(shape);
    a.x = x; a.res = residual; a.w = weight; a.gate = gate; a.y = y; a.h_out = h;
    return done(run_block_norm_fwd(shape->dtype, shape->stream_dtype != shape->dtype, shape->post_norm != 0, a, static_cast<hipStream_t>(hip_stream)));
}

int deltanet_block_norm_workspace_bytes(const dn_block_norm_shape *shape, size_t *out_bytes) {
    if (!out_bytes) return DN_ERR_NULL;
    if (int rc = check_block_norm(shape)) return rc;
    const int blocks = block_norm_bwd_blocks(shape->dtype, shape->T, shape->D);
    *out_bytes = blocks > 1 ? (size_t)blocks * 2 * shape->D * sizeof(float) : 0;
    return DN_OK;
}

int deltanet_block_norm_bwd(const dn_block_norm_shape *shape, const void *dy, const void *dh, const void *h, const void *x,
                            const void *weight, const void *gate, void *dx, void *dresidual, float *dweight, float *dgate,
                            void *workspace, size_t workspace_bytes, void *hip_stream) {
    size_t need = 0;
    if (int rc = deltanet_block_norm_workspace_bytes(shape, &need)) return rc;
    const bool branch = shape->post_norm || gate;
    if (branch) if (int rc = check_stride(shape->x_stride, shape->D, elem_bytes(shape->dtype))) return rc;
    if (shape->T && (!dy || !h || (branch && !x))) return DN_ERR_NULL;
    if (dgate && !gate) return DN_ERR_NULL;
    if (int rc = check_align({dy, dh, h, x, weight, gate, dx, dresidual, dweight, dgate, workspace})) return rc;
    const bool sums = dweight || dgate;
    if (sums && need && (!workspace || workspace_bytes < need)) return DN_ERR_WORKSPACE;
    BlockNormArgs a = block_norm_args(shape);
    a.dy = dy; a.dh = dh; a.h = h; a.x = x; a.w = weight; a.gate = gate;
    a.dx = dx; a.dres = dresidual; a.dw = dweight; a.dgate = dgate;
    a.partial = sums ? static_cast<float *>(workspace) : nullptr;
    return done(run_block_norm_bwd(shape->dtype, shape->stream_dtype != shape->dtype, shape->post_norm != 0, a, static_cast<hipStream_t>(hip_stream)));
}

} // extern "C"
