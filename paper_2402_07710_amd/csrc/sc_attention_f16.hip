// The attention kernels on f16 rows.
#include "sc_attention.h"

namespace sc {
int launch_attention_f16(const Attention& p, AttentionShape shape, hipStream_t s) { return launch_attention<SC_F16>(p, shape, s); }
int launch_attention_grad_f16(const Attention& p, bool alone, hipStream_t s) { return launch_attention_grad<SC_F16>(p, alone, s); }
}  // namespace sc
