// Kernel arguments and launch sequences of the operators around a layer's mixer (short convolution, output norm, block norm), shared by the C ABI
// (dn_layer_api.hip) and the kernels.
#pragma once
#include "dn_host.hpp"

namespace dn {

constexpr int kMostTaps = 4, kMostParts = 3;

struct ConvArgs {
    const void *x, *w, *b, *s0;          // s0: initial_state
    void *y[kMostParts], *sT;            // sT: final_state
    const void *dy[kMostParts], *dsT;
    void *dx, *ds0;
    float *partial;                      // backward: gradients of weight and bias per workgroup [blocks][C W + C] (workspace)
    float *dw, *db;
    const int32_t *cu;                   // packed: offsets on the device; else null
    long x_stride, dx_stride;            // elements
    int N, L, T, C, W;                   // N sequences (dense: of L rows each); T rows
    int at[kMostParts + 1];              // the parts' first channels, ending with C
    int silu;                            // bit p: part p is activated
};

struct OutNormArgs {
    const void *o, *gate, *w, *dy;
    void *y, *d_o, *dgate;
    float *partial, *dw;                 // backward: the weight's gradient per workgroup [blocks][d] (workspace)
    long o_stride, gate_stride, dgate_stride; // elements between tokens
    int T, H, act;
    unsigned magic;                      // row / H = mulhi(row, magic) >> shift
    int shift;
    float eps;
    bool once;                           // whether gradients are stored past the caches (set by the launch)
};

struct BlockNormArgs {
    const void *x, *res, *w, *gate, *dy, *h, *dh;
    void *y, *h_out, *dx, *dres;
    float *partial, *dw, *dgate;         // backward: gradients of weight and gate per workgroup [blocks][2 D] (workspace)
    long x_stride, res_stride;           // elements
    int T, D;
    float scale, res_scale, eps;
    bool once;                           // whether the stream and gradients are stored past the caches (set by the launch)
};

// All return 0 or the hipError_t of the failing launch.  dtype: 0 = fp32, 1 = bf16.
int run_short_conv_fwd(int dtype, const ConvArgs &a, hipStream_t stream);
int run_short_conv_bwd(int dtype, const ConvArgs &a, hipStream_t stream);
int run_out_norm_fwd(int dtype, int d, const OutNormArgs &a, hipStream_t stream);
int run_out_norm_bwd(int dtype, int d, const OutNormArgs &a, hipStream_t stream);
int run_block_norm_fwd(int dtype, bool wide_stream, bool post, const BlockNormArgs &a, hipStream_t stream);
int run_block_norm_bwd(int dtype, bool wide_stream, bool post, const BlockNormArgs &a, hipStream_t stream);

// Workgroups of the backward passes that leave partial sums of vectors' gradients (per block of columns: the convolution).
int short_conv_bwd_blocks(int dtype, const ConvArgs &a);
int out_norm_bwd_blocks(int dtype, int d, int T, int H);
int block_norm_bwd_blocks(int dtype, int T, int D);

// Sums `count` partial vectors of n elements, in an order that count and n decide (some threads an element, each with every so manieth vector, joined in turn): the first n1 of a vector go to out1, the others to out2 (null: not wanted).
int run_sum_partials(const float *partial, int count, long n, long n1, float *out1, float *out2, hipStream_t stream);

} // namespace dn
