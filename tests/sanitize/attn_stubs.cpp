// Stand-ins for the attention operators' launch sequences, as abi_stubs.cpp for the others: they record that they were reached and touch no pointer.
#include "../../paper_2406_06484_amd/csrc/dn_attn_host.hpp"

int g_attn_calls = 0;

namespace dn {
int run_norm_rope_fwd(int, int, const RowArgs &, hipStream_t) { ++g_attn_calls; return 0; }
int run_norm_rope_bwd(int, int, const RowArgs &, hipStream_t) { ++g_attn_calls; return 0; }
int run_paged_append(int, int, bool, bool, const RowArgs &, const PagedArgs &, hipStream_t) { ++g_attn_calls; return 0; }
int run_paged_read(int, int, bool, const RowArgs &, const PagedArgs &, hipStream_t) { ++g_attn_calls; return 0; }
size_t paged_attn_workspace(int, int, const AttnArgs &a) { return a.splits * 16u; }
int run_paged_attn(int, int, bool, const AttnArgs &, hipStream_t) { ++g_attn_calls; return 0; }
} // namespace dn
