// Attention of many queries over pages of codes (paged_tiles.h).
#include "paged_tiles.h"

namespace aquakv {

hipError_t launch_paged_tiles(int n_codewords, const PagedAttendArgs& a, hipStream_t stream) { return paged::launch_tiles<false>(n_codewords, a, stream); }

}  // namespace aquakv
