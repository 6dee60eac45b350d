// Attention over a paged cache: tiles of 16 rows (cache_attention.h).
#include "cache_attention.h"

namespace axe {

template <>
void launch_attention_narrow<1>(const CacheArgs& a, uint32_t groups, hipStream_t s) {
  if (a.groups) launch_attention<1, true>(a, groups, s);
  else launch_attention<1, false>(a, groups, s);
}

}  // namespace axe
