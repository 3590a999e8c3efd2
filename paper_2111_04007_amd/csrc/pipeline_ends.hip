// Launches of the embedding, the loss and the global gradient norm (see pipeline_ends.h).
#include "embedding.h"
#include "grad_clip.h"
#include "loss.h"

namespace varuna {

template hipError_t launch_embedding_fwd<float>(const EmbedArgs&, hipStream_t);
template hipError_t launch_embedding_fwd<bf16>(const EmbedArgs&, hipStream_t);
template hipError_t launch_embedding_bwd<float>(const EmbedGradArgs&, hipStream_t);
template hipError_t launch_embedding_bwd<bf16>(const EmbedGradArgs&, hipStream_t);
template hipError_t launch_cross_entropy<float>(const LossArgs&, hipStream_t);
template hipError_t launch_cross_entropy<bf16>(const LossArgs&, hipStream_t);

}  // namespace varuna
