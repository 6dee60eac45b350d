// Attention over a paged cache: tiles of 16 rows (cache_attention.h).
#include "cache_attention.h"

namespace axe {

template <>
void launch_attention_narrow<1>(const CacheArgs& a, hipStream_t s) {
  launch_attention<1, true>(a, a.groups, s);
}

}  // namespace axe
