// token_rows.h -- a token's row of the table (device code).
#pragma once

#include "token_ops.h"

namespace sw {
namespace embed {

// The token as a row of the table, or V where it is none.
__device__ __forceinline__ uint32_t row_of(const EmbedArgs& a, int64_t t) {
  const int64_t v = a.wide ? ((const int64_t*)a.tokens)[t] : ((const int32_t*)a.tokens)[t];
  return v >= 0 && v < a.V ? (uint32_t)v : (uint32_t)a.V;
}

}  // namespace embed
}  // namespace sw
