// Attention over fp32 latents.
#include "scd_latent_attend.h"

namespace scd {

hipError_t launch_latent_core_f32(const LatentAttendParams& p, hipStream_t stream) { return launch_latent_as<float>(p, stream); }

}  // namespace scd
