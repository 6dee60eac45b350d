// Attention over a paged cache: tiles of 32 rows (cache_attention.h).
#include "cache_attention.h"

namespace axe {

template <>
void launch_attention_narrow<2>(const CacheArgs& a, hipStream_t s) {
  launch_attention<2, true>(a, a.groups, s);
}

}  // namespace axe
