// Kernel arguments and launch sequences of the attention operators, shared by the C ABI (dn_attn_api.hip) and the kernels.
#pragma once
#include "dn_host.hpp"

namespace dn {

// Rows of q, k (and v) to normalise, rotate, quantise or copy; what a caller leaves out is null.
struct RowArgs {
    const void *q, *k, *v;               // inputs, row strides below
    const void *qw, *kw;                 // RMS weights [d] in the element type
    const float *cs;                     // cos | sin table [max_pos][rot]
    const int32_t *positions;            // [T]; or null: t % seq_len, or the place in the sequence where there is a cache
    void *q_out, *k_out, *v_out;         // contiguous
    const void *dq_out, *dk_out;         // backward: gradients with respect to q_out, k_out (contiguous)
    float *partial;                      // backward: weights' gradients per workgroup [blocks][2][d] (workspace)
    float *dqw, *dkw;
    long q_stride, k_stride, v_stride;   // elements
    int T, Hq, Hkv;
    int rot, interleaved, max_pos, seq_len;
    float eps;
};

// The cache and the batch's place in it.
struct PagedArgs {
    void *kp, *vp;
    float *ks, *vs;                      // 4-bit pages: the groups' factors, a byte each
    const int32_t *cu, *kv_len, *table;  // cu: of the rows that are written, read back or attend
    int N, page_shift, num_pages, max_pages, max_kv;
    bool fp4;                            // pages of e2m1 numbers
};

struct AttnArgs {
    RowArgs r;                           // q, q_out, strides, T, heads
    PagedArgs c;
    float scale;
    int window, max_q;
    int splits;                          // most splits of any row (the workspace's layout)
    int zero_front, zero_rest;           // whether rows in front of the first sequence, past the last one, are this launch's to zero
    void *workspace;
};

// All return 0 or the hipError_t of the failing launch.  dtype: 0 = fp32, 1 = bf16; fp8: whether the pages are 8-bit (4-bit: fp4 in the arguments; else they have the tensors' type).
int run_norm_rope_fwd(int dtype, int d, const RowArgs &a, hipStream_t stream);
int run_norm_rope_bwd(int dtype, int d, const RowArgs &a, hipStream_t stream);
int run_paged_append(int dtype, int d, bool fp8, bool norm, const RowArgs &a, const PagedArgs &c, hipStream_t stream);
int run_paged_read(int dtype, int d, bool fp8, const RowArgs &a, const PagedArgs &c, hipStream_t stream);
size_t paged_attn_workspace(int dtype, int d, const AttnArgs &a);
int run_paged_attn(int dtype, int d, bool fp8, const AttnArgs &a, hipStream_t stream);

// Workgroups of the backward pass per tensor: each leaves one partial sum of the weight's gradient.
inline int norm_rope_bwd_blocks(int T) {
    const int blocks = (T + 3) / 4;
    return blocks < 512 ? blocks : 512;
}

} // namespace dn
