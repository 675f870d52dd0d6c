// linear_walk_f32.hip -- the chunked walks of linear attention on fp32 inputs.
#include "linear_walk.h"

namespace sw {
namespace lin {
int launch_walk_f32(const WalkArgs& a, Mode m, int nt, hipStream_t st) {
  return launch_walk<F32>(a, m, nt, st);
}
}  // namespace lin
}  // namespace sw
