// Attention for trees of drafted tokens: the kernels of attention over pages, whose rows see of the queries' own tokens those that their bits say.
// Bits are looked at in tiles that reach behind the tokens ahead of the drafts, eight (or four) of them at once, from two words.  Trees have a few dozen rows a kv head, where attention's
// own calls have one query or a chunk: waves of 48 rows, row tiles spread over the chip and pieces of equal size over all sequences are theirs (the rules are with the plan).
// 26 drafts of 4 heads a kv head over 2000 tokens 16.8 us (13.8 in the first kernel, a chain of waits, and 4 to join); 12 drafts over 32 x 8000 tokens, uniform 4 bits,
// 136 us (1.6 TB/s: vector pipes busy in 58 % of the cycles, two waves a SIMD); 64 over 4 x 16 384, 64 points, 96 us (560 TFLOP/s of 1200 that a library product reaches).
#include "paged_rows.h"
#include "paged_tiles.h"

namespace aquakv {

hipError_t launch_paged_tree_rows(int dtype, int n_codewords, int cols, dim3 blocks, const PagedAttendArgs& a, hipStream_t stream) {
  return paged::launch_rows<true>(dtype, n_codewords, cols, blocks, a, stream);
}
hipError_t launch_paged_tree_tiles(int n_codewords, const PagedAttendArgs& a, hipStream_t stream) { return paged::launch_tiles<true>(n_codewords, a, stream); }

}  // namespace aquakv
