// Attention over fp32 latents.
#include "scd_latent_attend.h"

namespace scd {

hipError_t launch_latent_core_f32(const LatentAttendParams& p, hipStream_t stream) {
  if (p.cache.latent <= 64) return launch_latent_shape<float, 64, 1>(p, stream);
  if (p.cache.latent <= 128) return launch_latent_shape<float, 128, 1>(p, stream);
  if (p.cache.latent <= 256) return launch_latent_shape<float, 256, 1>(p, stream);
  return launch_latent_shape<float, 512, 1>(p, stream);
}

}  // namespace scd
