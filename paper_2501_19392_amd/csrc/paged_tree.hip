// Attention for trees of drafted tokens: the kernels of attention over pages, whose rows see of the queries' own tokens those that their bits say.
#include "paged_rows.h"
#include "paged_tiles.h"

namespace aquakv {

hipError_t launch_paged_tree_rows(int dtype, int n_codewords, int cols, dim3 blocks, const PagedAttendArgs& a, hipStream_t stream) {
  return paged::launch_rows<true>(dtype, n_codewords, cols, blocks, a, stream);
}
hipError_t launch_paged_tree_tiles(int n_codewords, const PagedAttendArgs& a, hipStream_t stream) { return paged::launch_tiles<true>(n_codewords, a, stream); }

}  // namespace aquakv
