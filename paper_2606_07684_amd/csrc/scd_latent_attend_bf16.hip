// Attention over bf16 latents.
#include "scd_latent_attend.h"

namespace scd {

hipError_t launch_latent_core_bf16(const LatentAttendParams& p, hipStream_t stream) {
  const bool two = p.plan.rows == 128;
  if (p.cache.latent <= 64)
    return two ? launch_latent_shape<uint16_t, 64, 2>(p, stream) : launch_latent_shape<uint16_t, 64, 1>(p, stream);
  if (p.cache.latent <= 128)
    return two ? launch_latent_shape<uint16_t, 128, 2>(p, stream) : launch_latent_shape<uint16_t, 128, 1>(p, stream);
  if (p.cache.latent <= 256) return launch_latent_shape<uint16_t, 256, 1>(p, stream);
  return launch_latent_shape<uint16_t, 512, 1>(p, stream);
}

}  // namespace scd
