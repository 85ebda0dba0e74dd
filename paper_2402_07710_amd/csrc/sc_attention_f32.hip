// The attention kernels on f32 rows.
#include "sc_attention.h"

namespace sc {
int launch_attention_f32(const Attention& p, AttentionShape shape, hipStream_t s) { return launch_attention<SC_F32>(p, shape, s); }
int launch_attention_grad_f32(const Attention& p, bool alone, hipStream_t s) { return launch_attention_grad<SC_F32>(p, alone, s); }
}  // namespace sc
