// Calls the C ABI of the attention operators (host layer alone, launches replaced by stand-ins) under AddressSanitizer / UndefinedBehaviorSanitizer:
// refusals, sizes at the ends of their ranges, and calls that pass.  Device pointers are fakes that nothing dereferences.
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "../../include/deltanet.h"

extern int g_attn_calls;

#define EXPECT(cond)                                                          \
    do {                                                                      \
        if (!(cond)) { printf("FAILED line %d: %s\n", __LINE__, #cond); return 1; } \
    } while (0)

int main() {
    void *f = (void *)0x1000;
    float *ff = (float *)f;
    const int32_t *fi = (const int32_t *)f;
    size_t bytes = 0;
    dn_qk_shape q = {8, 4, 2, 64, DN_BF16, 8, 256, 128};
    dn_rope r = {64, 0, 16, 1e-6f};
    EXPECT(deltanet_qk_norm_rope_fwd(&q, &r, f, f, f, f, ff, fi, f, f, nullptr) == DN_OK);
    EXPECT(deltanet_qk_norm_rope_workspace_bytes(&q, &bytes) == DN_OK && bytes == 2 * 2 * 64 * 4);
    EXPECT(deltanet_qk_norm_rope_bwd(&q, &r, f, f, f, f, nullptr, nullptr, ff, nullptr, f, f, nullptr, nullptr, nullptr, 0, nullptr) == DN_OK);
    EXPECT(deltanet_qk_norm_rope_bwd(&q, &r, f, f, f, f, f, f, ff, nullptr, f, f, ff, ff, f, bytes - 1, nullptr) == DN_ERR_WORKSPACE);
    for (int32_t big : {INT32_MAX, INT32_MIN, 1 << 30}) {
        dn_qk_shape b = q;
        b.T = big;
        EXPECT(deltanet_qk_norm_rope_workspace_bytes(&b, &bytes) == DN_ERR_SHAPE);
        b = q; b.Hq = big;
        EXPECT(deltanet_qk_norm_rope_workspace_bytes(&b, &bytes) == DN_ERR_SHAPE);
        b = q; b.q_stride = (int64_t)big * 1024;
        EXPECT(deltanet_qk_norm_rope_workspace_bytes(&b, &bytes) == DN_ERR_SHAPE);
    }
    dn_paged_shape p;
    memset(&p, 0, sizeof(p));
    p.num_seqs = 2; p.T = 8; p.Hq = 4; p.Hkv = 2; p.d = 64; p.dtype = p.cache_dtype = DN_BF16;
    p.page_size = 16; p.num_pages = 9; p.max_pages = 4; p.max_q = 8; p.max_kv = 64;
    p.cu_q = p.kv_len = p.page_table = fi;
    p.q_stride = 256; p.k_stride = p.v_stride = 128;
    dn_paged_cache c = {f, f, nullptr, nullptr};
    EXPECT(deltanet_paged_append(&p, f, f, &c, nullptr) == DN_OK);
    EXPECT(deltanet_paged_norm_rope_append(&p, &r, f, f, f, nullptr, nullptr, ff, f, &c, nullptr) == DN_OK);
    EXPECT(deltanet_paged_read(&p, &c, fi, 5, f, f, nullptr) == DN_OK);
    EXPECT(deltanet_paged_attn_workspace_bytes(&p, 0, &bytes) == DN_OK);
    EXPECT(deltanet_paged_attn_fwd(&p, f, &c, 0.125f, INT32_MAX, f, f, 1 << 20, nullptr) == DN_OK);
    EXPECT(g_attn_calls == 6);
    dn_paged_shape b = p;
    b.max_pages = INT32_MAX; b.max_kv = (1 << 30) + 1;
    EXPECT(deltanet_paged_attn_workspace_bytes(&b, 0, &bytes) == DN_ERR_SHAPE);
    b.max_kv = 1 << 30;
    EXPECT(deltanet_paged_attn_workspace_bytes(&b, 0, &bytes) == DN_OK);
    b = p; b.page_size = 0;
    EXPECT(deltanet_paged_append(&b, f, f, &c, nullptr) == DN_ERR_UNSUPPORTED);
    b = p; b.page_size = 256; b.Hq = b.Hkv = 8192; b.d = 256; b.T = b.max_q = 1;
    EXPECT(deltanet_paged_attn_workspace_bytes(&b, 0, &bytes) == DN_ERR_SHAPE); // a page of 1 GiB
    EXPECT(deltanet_paged_attn_fwd(&p, f, &c, NAN, 0, f, f, 1 << 20, nullptr) == DN_ERR_SHAPE);
    EXPECT(deltanet_paged_attn_fwd(&p, f, nullptr, 1.f, 0, f, f, 1 << 20, nullptr) == DN_ERR_NULL);
    EXPECT(g_attn_calls == 6);
    printf("attention host layer under sanitizers: ok\n");
    return 0;
}
