// The tiled products of the gated feed-forward block for float32 operands, each three bfloat16 limbs.
#include "gated_ff_tiles.cuh"

namespace ff {

int32_t launch_tiles_f32(Kind kind, bool pair, const Maps& maps, const Args& args, int device, int sms, cudaStream_t st) {
#define GNNCO_FF(KIND) \
  case KIND: return pair ? launch_one<KIND, 3, true>(maps, args, device, sms, st) : launch_one<KIND, 3, false>(maps, args, device, sms, st)
  switch (kind) {
    GNNCO_FF(kGlu);
    GNNCO_FF(kGluBack);
    GNNCO_FF(kDown);
    GNNCO_FF(kDx);
    GNNCO_FF(kWeights);
  }
#undef GNNCO_FF
  return GNNCO_INTERNAL;
}

}  // namespace ff
