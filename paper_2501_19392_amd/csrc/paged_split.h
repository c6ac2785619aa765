// How attention over pages cuts tokens into pieces of whole tiles: arithmetic alone, on the device and wherever else it is compiled.
// Sums are of tiles, of which there are below 2^27 in a sequence and 2^31 in a batch: a piece's end in tokens can pass 2^31.
#pragma once
#include <cstdint>

namespace aquakv {
namespace paged {

// tiles of a sequence, or what of it is seen (nothing: 0 or fewer tokens)
constexpr int tiles_of_tokens(int tokens, int tile) { return tokens > 0 ? (tokens - 1) / tile + 1 : 0; }

// The tokens of a piece, one of equal pieces of `each` tiles, as far as there are some: empty otherwise.
struct TokenRange { int begin, end; };
constexpr TokenRange piece_range(int piece, int each, int tile, int tokens) {
  const int tiles = tiles_of_tokens(tokens, tile), first = piece * each;
  if (first >= tiles) return {0, 0};
  return {first * tile, tiles - first > each ? (first + each) * tile : tokens};
}

// whole pieces that all tiles together may make
constexpr int piece_room(int slots, int batch) {
  const int half = slots / 2 > 1 ? slots / 2 : 1;
  return slots - batch > half ? slots - batch : half;
}
// tiles per piece with which ceil(tiles / piece) over all sequences is at most max(slots, slots / 2 + batch), whatever the lengths
constexpr int piece_tiles(int total, int slots, int batch) {
  const uint32_t room = (uint32_t)piece_room(slots, batch);
  return (int)(((uint32_t)total + room - 1) / room);
}
// Pieces of sequences that are in more than one, at most: x tiles in pieces of n < x are ceil(x / n) < 2 x / n of them, and total / n <= room.
constexpr int piece_results(int slots, int batch) { return 2 * piece_room(slots, batch); }
// Short pieces make half as many: two waves of one tile take as long as one of two, whose results are half as many to write and to join (one query of
// 10 000 tokens, 313 tiles: 20.0 us in pieces of one tile, 15.9 of two; of 6000 14.9, 14.6; 5 queries of 2000 tokens of 8 sequences: 20.5 in pieces of two, 18.6 of
// three, 19.7 of four).  Longer ones want all waves there are (32 x 16 384 tokens: 95 us, on half of the waves 111).
constexpr int short_piece(int total, int slots) {
  const uint32_t half = (uint32_t)(slots / 2 > 1 ? slots / 2 : 1), each = ((uint32_t)total + half - 1) / half;
  return (int)(each < 4u ? each : 4u);
}

}  // namespace paged
}  // namespace aquakv
