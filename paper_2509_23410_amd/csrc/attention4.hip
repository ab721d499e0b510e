// The attention's launches for cells of 4 bits (patch_attention4).
#include "attention_kernels.h"

namespace patch {

void launch_attention4(const AttnArgs& a, hipStream_t stream) { launch_cells<kE2m1>(a, stream); }

}  // namespace patch
