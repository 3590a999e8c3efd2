// Launches of rotary positions, the residual norms and AdamW (see layer_ops.h).
#include "adamw.h"
#include "residual_norm.h"
#include "rotary.h"

namespace varuna {

template hipError_t launch_rotary<float>(const RotaryArgs&, hipStream_t);
template hipError_t launch_rotary<bf16>(const RotaryArgs&, hipStream_t);
template hipError_t launch_residual_norm_fwd<float>(const NormArgs&, hipStream_t);
template hipError_t launch_residual_norm_fwd<bf16>(const NormArgs&, hipStream_t);
template hipError_t launch_residual_norm_bwd<float>(const NormArgs&, hipStream_t);
template hipError_t launch_residual_norm_bwd<bf16>(const NormArgs&, hipStream_t);

}  // namespace varuna
