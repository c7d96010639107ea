// Calls the C ABI of the layer operators (host layer alone, launches replaced by stand-ins) under AddressSanitizer / UndefinedBehaviorSanitizer: refusals, sizes at the ends of
// their ranges, and calls that pass.  Device pointers are fakes that nothing dereferences.
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include "../../include/deltanet.h"

extern int g_layer_calls;

#define EXPECT(cond)                                                          \
    do {                                                                      \
        if (!(cond)) { printf("FAILED line %d: %s\n", __LINE__, #cond); return 1; } \
    } while (0)

int main() {
    void *f = (void *)0x1000;
    float *ff = (float *)f;
    size_t bytes = 1;
    void *one[1] = {f}, *three[3] = {f, f, f};
    const void *c3[3] = {f, f, f};
    dn_conv_shape c = {1, 16, 64, 4, DN_BF16, 0, nullptr, nullptr, 1, {64, 0, 0}, {1, 0, 0}, 64, 64};
    EXPECT(deltanet_short_conv_fwd(&c, f, f, nullptr, nullptr, one, nullptr, nullptr) == DN_OK); // (an array of as many pointers as there are parts)
    int32_t cu[3] = {0, 5, 16};
    c.cu_seqlens = (const int32_t *)f; c.cu_seqlens_host = cu; c.num_seqs = 2;
    c.parts = 3; c.width[0] = 16; c.width[1] = 16; c.width[2] = 32;
    EXPECT(deltanet_short_conv_fwd(&c, f, f, f, f, three, f, nullptr) == DN_OK);
    EXPECT(deltanet_short_conv_workspace_bytes(&c, &bytes) == DN_OK && bytes == 0);
    EXPECT(deltanet_short_conv_bwd(&c, f, f, c3, f, f, f, f, ff, ff, f, nullptr, 0, nullptr) == DN_OK);
    cu[1] = 17;
    EXPECT(deltanet_short_conv_fwd(&c, f, f, f, f, three, f, nullptr) == DN_ERR_CUSEQLENS);
    c.cu_seqlens = nullptr;
    for (int32_t big : {INT32_MAX, INT32_MIN, (1 << 30) + 1}) {
        dn_conv_shape b = c;
        b.L = big;
        EXPECT(deltanet_short_conv_workspace_bytes(&b, &bytes) == DN_ERR_SHAPE);
        b = c; b.B = big;
        EXPECT(deltanet_short_conv_workspace_bytes(&b, &bytes) == DN_ERR_SHAPE);
        b = c; b.C = big;
        EXPECT(deltanet_short_conv_workspace_bytes(&b, &bytes) == DN_ERR_SHAPE);
        b = c; b.width[2] = big;
        EXPECT(deltanet_short_conv_workspace_bytes(&b, &bytes) == DN_ERR_SHAPE);
        b = c; b.x_stride = (int64_t)big * 1024;
        EXPECT(deltanet_short_conv_workspace_bytes(&b, &bytes) == DN_ERR_SHAPE);
        b = c; b.W = big;
        EXPECT(deltanet_short_conv_workspace_bytes(&b, &bytes) == DN_ERR_UNSUPPORTED);
    }
    dn_out_norm_shape o = {200, 4, 64, DN_BF16, DN_ACT_SILU, 1e-6f, 256, 256, 256};
    EXPECT(deltanet_out_norm_fwd(&o, f, f, f, f, nullptr) == DN_OK);
    EXPECT(deltanet_out_norm_workspace_bytes(&o, &bytes) == DN_OK && bytes == 2 * 64 * 4);
    EXPECT(deltanet_out_norm_bwd(&o, f, f, f, f, f, f, ff, f, bytes, nullptr) == DN_OK);
    for (int32_t H : {1, 2, 3, 8191, INT32_MAX / 256}) { // (divisors of every size)
        dn_out_norm_shape b = o;
        b.H = H; b.T = 1; b.o_stride = b.gate_stride = (int64_t)H * 64 < (1ll << 31) ? (int64_t)H * 64 : 0;
        EXPECT(deltanet_out_norm_fwd(&b, f, f, f, f, nullptr) == DN_OK);
    }
    dn_block_norm_shape k = {200, 64, DN_BF16, DN_F32, 1, 0.5f, 1.f, 1e-6f, 64, 64};
    EXPECT(deltanet_block_norm_fwd(&k, f, f, f, f, f, f, nullptr) == DN_OK);
    EXPECT(deltanet_block_norm_workspace_bytes(&k, &bytes) == DN_OK && bytes == 2 * 2 * 64 * 4);
    EXPECT(deltanet_block_norm_bwd(&k, f, f, f, f, f, f, f, f, ff, ff, f, bytes, nullptr) == DN_OK);
    k.scale = NAN;
    EXPECT(deltanet_block_norm_fwd(&k, f, f, f, f, f, f, nullptr) == DN_ERR_SHAPE);
    EXPECT(g_layer_calls == 12);
    printf("layer host layer under sanitizers: ok\n");
    return 0;
}
