// The attention kernels on bf16 rows.
#include "sc_attention.h"

namespace sc {
int launch_attention_bf16(const Attention& p, AttentionShape shape, hipStream_t s) { return launch_attention<SC_BF16>(p, shape, s); }
int launch_attention_grad_bf16(const Attention& p, bool alone, hipStream_t s) { return launch_attention_grad<SC_BF16>(p, alone, s); }
}  // namespace sc
