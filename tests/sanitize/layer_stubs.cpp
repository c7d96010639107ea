// Stand-ins for the layer operators' launch sequences, as attn_stubs.cpp for the attention's: they record that they were reached and touch no pointer.
#include "../../paper_2406_06484_amd/csrc/dn_layer_host.hpp"

int g_layer_calls = 0;

namespace dn {
int run_short_conv_fwd(int, const ConvArgs &, hipStream_t) { ++g_layer_calls; return 0; }
int run_short_conv_bwd(int, const ConvArgs &, hipStream_t) { ++g_layer_calls; return 0; }
int run_out_norm_fwd(int, int, const OutNormArgs &, hipStream_t) { ++g_layer_calls; return 0; }
int run_out_norm_bwd(int, int, const OutNormArgs &, hipStream_t) { ++g_layer_calls; return 0; }
int run_block_norm_fwd(int, bool, bool, const BlockNormArgs &, hipStream_t) { ++g_layer_calls; return 0; }
int run_block_norm_bwd(int, bool, bool, const BlockNormArgs &, hipStream_t) { ++g_layer_calls; return 0; }
int short_conv_bwd_blocks(int, const ConvArgs &a) { return a.T > 100 ? 2 : 1; }
int out_norm_bwd_blocks(int, int, int T, int) { return T > 100 ? 2 : 1; }
int block_norm_bwd_blocks(int, int T, int) { return T > 100 ? 2 : 1; }
} // namespace dn
