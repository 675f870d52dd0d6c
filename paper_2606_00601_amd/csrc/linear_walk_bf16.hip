// linear_walk_bf16.hip -- the chunked walks of linear attention on bf16 inputs.
#include "linear_walk.h"

namespace sw {
namespace lin {
int launch_walk_bf16(const WalkArgs& a, Mode m, int nt, hipStream_t st) {
  return launch_walk<Bf16>(a, m, nt, st);
}
}  // namespace lin
}  // namespace sw
