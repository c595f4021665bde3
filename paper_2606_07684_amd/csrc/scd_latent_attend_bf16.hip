// Attention over bf16 latents.
#include "scd_latent_attend.h"

namespace scd {

hipError_t launch_latent_core_bf16(const LatentAttendParams& p, hipStream_t stream) { return launch_latent_as<uint16_t>(p, stream); }

}  // namespace scd
