// What the kernels that attend over pages of codes share: which rows and tokens they take, codes to fp16 operands of the matrix
// instructions, the query's way in and the result's way out.
//
// Precision.  Operands are fp16 (11 bits): the rotated query times a power of two of its own, grid points times a power of two of
// the grid's, weights times the token's scale relative to a running reference, all sums fp32.  fp32 layers hold each of them as two
// fp16 numbers (22 bits) and take three products.  Uniform codes and zero points are exact operands: a code at the low end of a half-word is the
// subnormal fp16 number code * 2^-24, which the matrix instructions take as it is, so that a mask is all the conversion there is.  They align such products
// by the exponent, 10 above the code's bits, so that a sum keeps 2^-17 of its largest one, far below the rounding of query and weights; fp32 layers, and
// paged_tiles.hip, which converts codes once for many rows, make them normal numbers, whose sums are fp32's.
//
// fp16 ends at 2^-24: coordinates of a query below 2^-27 of its largest (uniform codes, which are masked in place: 2^-23, 2 bits 2^-21), and weights with their
// scales below 2^-22 of the largest that scores and scales of a tile allow (each for itself: a weight's token may have a smaller scale than its neighbours), have
// fewer bits than 11, down to 2^-38 (2^-34, 2^-32) and 2^-33.
#pragma once
#include "codec_core.h"
#include "kernels.h"
#include "paged_split.h"

namespace aquakv {
namespace paged {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef const __attribute__((address_space(4))) int32_t* ConstInts;       // (scalar loads: what is read through it is not written meanwhile)
inline __device__ ConstInts const_ints(const int32_t* p) { return (ConstInts)(uintptr_t)p; }

constexpr int kTile = 32;                    // tokens of a tile: four groups of 8, each within a page
constexpr int kTileWaves = 8, kTileRows = 32 * kTileWaves;  // of a workgroup of paged_tiles
constexpr int kQueryExp = 14;                // largest coordinate of a row's query: 2^13 ... 2^14
constexpr float kTopExp = 15.0f, kTopWeight = 0x1p15f;      // a weight beyond 2^kTopExp moves the reference,
constexpr float kStartExp = 8.0f;            // so that the largest is 2^kStartExp: what is 2^-33 of it still counts

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// ---------------------------------------------------------------- rows, pieces
// What a sequence asks: `count` queries, its last tokens, rows first ... of q, of which n are answered; len tokens are cached.
struct PagedQueries { int64_t first; int count, n, len; };
__device__ __forceinline__ int length_of(const PagedAttendArgs& a, int len) {
  return (int)min((int64_t)max(len, 0), (int64_t)a.table_pages * a.pool.page_tokens);
}
__device__ __forceinline__ PagedQueries paged_queries(const PagedAttendArgs& a, int b) {
  PagedQueries w;
  w.first = (int64_t)b * a.max_queries;
  w.count = a.max_queries;
  if (a.q_start != nullptr) {
    const int64_t from = const_ints(a.q_start)[b], to = const_ints(a.q_start)[b + 1];
    w.first = from < 0 ? 0 : from < a.q_rows ? from : a.q_rows;
    const int64_t end = to < w.first ? w.first : to < a.q_rows ? to : a.q_rows;
    w.count = (int)(end - w.first);
  }
  w.count = uniform(w.count);
  w.n = min(w.count, a.max_queries);
  w.len = length_of(a, const_ints(a.seq_lens)[b]);
  return w;
}

// The tokens of all sequences are cut into pieces of equally many tiles, so that about a.slots of them cover the batch whatever its
// lengths (each sequence has one at least): item i of the launch is piece `piece` of `pieces` of sequence b (-1: behind the last).
// RESULTS: `results` is the number of pieces ahead of this sequence's that are not the only one of theirs.
struct Share { int b, piece, pieces, tiles, items, results; };
template <int TILE> __device__ __forceinline__ int tiles_of(const PagedAttendArgs& a, int b) {
  return b < a.batch ? max(tiles_of_tokens(length_of(a, a.seq_lens[b]), TILE), 1) : 0;
}
// sums over the lanes up to and with this one
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111 /* row_shr:1 */, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142 /* row_bcast:15 */, 0xa, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x143 /* row_bcast:31 */, 0xc, 0xf, false);
  return x;
}
template <int TILE = kTile, bool RESULTS = false> __device__ __forceinline__ Share share_of(const PagedAttendArgs& a, int lane, int item) {
  Share s = {-1, 0, 1, 0, 0, 0};
  if (a.batch == 1) {
    const int n = max(tiles_of_tokens(length_of(a, const_ints(a.seq_lens)[0]), TILE), 1);
    s.tiles = max((n + a.slots - 1) / a.slots, short_piece(n, a.slots));
    s.items = s.pieces = (n + s.tiles - 1) / s.tiles;
    if (item < s.items) { s.b = 0; s.piece = item; }
    return s;
  }
  int total = 0;                                           // (all sequences' room is below 2^30 tiles)
  int tiles = 0;
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    tiles = tiles_of<TILE>(a, b0 + lane);
    total += __builtin_amdgcn_readlane(wave_scan(tiles), 63);
  }
  s.tiles = piece_tiles(total, a.slots, a.batch);
  // The fewest tiles that do, where a wave has all lengths: 32 x 16 384 tokens are 512 pieces of 32 tiles then, not 480 of 35 (94.3 us for 95.6).
  if (a.batch <= 64 && 2 * a.batch <= a.slots) {
    int low = max((int)(((uint32_t)total + a.slots - 1) / a.slots), 1);
    while (low < s.tiles) {
      const int mid = (low + s.tiles) >> 1;
      if (__builtin_amdgcn_readlane(wave_scan((int)(((uint32_t)tiles + mid - 1) / (uint32_t)mid)), 63) <= a.slots) s.tiles = mid;
      else low = mid + 1;
    }
  }
  s.tiles = max(s.tiles, short_piece(total, a.slots));
  int results = 0;
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    if (a.batch > 64) tiles = tiles_of<TILE>(a, b0 + lane);
    const int mine = (int)((uint32_t)(tiles + s.tiles - 1) / (uint32_t)s.tiles);
    const int end = s.items + wave_scan(mine);             // items up to and with this sequence
    const uint64_t past = __builtin_amdgcn_ballot_w64(end > item);
    const int held = RESULTS ? results + wave_scan(mine > 1 ? mine : 0) : 0;      // results up to and with this sequence
    if (past != 0 && s.b < 0) {
      const int l = __builtin_ctzll(past);
      s.b = b0 + l;
      s.pieces = __builtin_amdgcn_readlane(mine, l);
      if constexpr (RESULTS) s.results = __builtin_amdgcn_readlane(held, l) - (s.pieces > 1 ? s.pieces : 0);
      s.piece = item - (__builtin_amdgcn_readlane(end, l) - s.pieces);
    }
    s.items = __builtin_amdgcn_readlane(end, 63);
    if constexpr (RESULTS) results = __builtin_amdgcn_readlane(held, 63);
  }
  s.b = uniform(s.b); s.piece = uniform(s.piece); s.pieces = uniform(s.pieces); s.tiles = uniform(s.tiles); s.items = uniform(s.items); s.results = uniform(s.results);
  return s;
}

// Which of up to eight consecutive tokens a row sees: the first n, or (drafts of a tree) those whose bit is set.
template <bool TREE> struct SeenOf {
  int n;
  __device__ __forceinline__ bool has(int e) const { return e < n; }
  __device__ __forceinline__ void keep(u32x4& w) const {   // half-words of the others become 0
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] &= (has(2 * i) ? 0xffffu : 0u) | (has(2 * i + 1) ? 0xffff0000u : 0u);
  }
};
template <> struct SeenOf<true> {
  uint32_t bits;
  __device__ __forceinline__ bool has(int e) const { return (bits >> e) & 1; }
  __device__ __forceinline__ void keep(u32x4& w) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] &= (has(2 * i) ? 0xffffu : 0u) | (has(2 * i + 1) ? 0xffff0000u : 0u);
  }
};
__device__ __forceinline__ uint32_t first_bits(int n) { return n >= 8 ? 255u : n <= 0 ? 0u : (1u << n) - 1u; }
// Bits draft ... draft + 7 of query row `row` of a tree: tokens ahead of the drafts (below 0) are seen, drafts behind the row's words are not.
__device__ __forceinline__ uint32_t tree_bits(const PagedAttendArgs& a, int64_t row, int draft) {
  if (draft <= -8) return 255u;
  const uint32_t* const words = a.tree + row * a.tree_words;
  const int at = draft >> 5;                               // (-1: ahead of the first)
  const uint32_t lo = at < 0 ? 0xffffffffu : at < a.tree_words ? words[at] : 0u, hi = at + 1 < a.tree_words ? words[at + 1] : 0u;
  return __builtin_amdgcn_alignbit(hi, lo, (uint32_t)draft & 31u) & 255u;
}

// Pool rows at which the four groups of 8 tokens of a tile start, -1: not there.
struct Rows { int r[4]; };
__device__ __forceinline__ Rows rows_of(const PagedAttendArgs& a, int b, int t) {
  const ConstInts table = const_ints(a.page_table) + (int64_t)b * a.table_pages;
  Rows out;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t group = (uint32_t)t / 8 + j;
    uint32_t page = (uint32_t)(((uint64_t)group * a.page_magic) >> 32), in = group - page * a.page_groups;      // (one short at most)
    if (in >= a.page_groups) { ++page; in -= a.page_groups; }
    const int at = page < (uint32_t)a.table_pages ? table[page] : -1;
    out.r[j] = (uint32_t)at < (uint32_t)a.pool.n_pages ? at * a.pool.page_tokens + (int)in * 8 : -1;
  }
  return out;
}
__device__ __forceinline__ unsigned there_of(const Rows& r) {
  return (r.r[0] >= 0) | (r.r[1] >= 0) << 1 | (r.r[2] >= 0) << 2 | (r.r[3] >= 0) << 3;
}
__device__ __forceinline__ int pick_of(const Rows& r, int j) {
  const int r0 = r.r[0], r1 = r.r[1], r2 = r.r[2], r3 = r.r[3];           // (values: a choice between elements would be one between addresses)
  const int lo = (j & 1) ? r1 : r0, hi = (j & 1) ? r3 : r2;
  return (j & 2) ? hi : lo;
}
__device__ __forceinline__ uint32_t row_of(const Rows& r, int j) { return (uint32_t)max(pick_of(r, j), 0); }      // a row there is, in any case

// ---------------------------------------------------------------- columns: lanes l, l ^ 16, l ^ 32, l ^ 48
__device__ __forceinline__ float column_max(float x) {
  float y = x;
  swap_lanes<16>(x, y);
  x = fmaxf(x, y);
  y = x;
  swap_lanes<32>(x, y);
  return fmaxf(x, y);
}
// a tile's weights, by pairs: one after the other, a lane's millions of equal weights would be off by 2^-24 of the sum each, all to one side (2^21 tokens: 1.2 %)
template <int N> __device__ __forceinline__ float sum_of(const float (&x)[N]) {
  float y[N / 2];
#pragma unroll
  for (int i = 0; i < N / 2; ++i) y[i] = x[2 * i] + x[2 * i + 1];
  if constexpr (N == 2) return y[0];
  else return sum_of(y);
}
__device__ __forceinline__ float column_sum(float x) { return far_sum<32>(far_sum<16>(x)); }
// The (unnormalised) transform of a row's 128 values, 32 g ... in lane group g.
__device__ __forceinline__ void wht_columns(float (&v)[32]) {
#pragma unroll
  for (int h = 1; h < 32; h <<= 1) {
#pragma unroll
    for (int r = 0; r < 32; ++r) {
      if ((r & h) == 0) {
        const float x = v[r], y = v[r + h];
        v[r] = x + y;
        v[r + h] = x - y;
      }
    }
  }
  wht_swap_stage<16>(v);
  wht_swap_stage<32>(v);
}

// The same transform of bf16 numbers (b[s]: values 8 s ... of the lane's 32) on the matrix cores, added to x: 32 instructions where the butterflies are 450,
// which a wave that has little else to do runs once, from a cold instruction cache.  H = +-1 is made from the lane's number: row m of product R is
// coordinate 32 (m / 4) + 4 R + m % 4, so that a lane ends with the coordinates it came with.
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
__device__ __forceinline__ void hadamard_columns(const bf16x8 (&b)[4], f32x4 (&x)[8], int lane) {
  const uint32_t m = lane & 15, g = lane >> 4, flip = 0x80008000u;
  const uint32_t p = 0x3f803f80u ^ ((m & 1) << 31) ^ ((__builtin_popcount((m >> 2) & g) & 1) ? flip : 0u), q = p ^ ((m & 2) ? flip : 0u);
  const u32x4 rows[4] = {{p, q, p, q}, {p, q, p ^ flip, q ^ flip}, {p ^ flip, q ^ flip, p ^ flip, q ^ flip}, {p ^ flip, q ^ flip, p, q}};
#pragma unroll
  for (int s = 0; s < 4; ++s)
#pragma unroll
    for (int R = 0; R < 8; ++R)
      x[R] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, rows[(R & 1) + 2 * (__builtin_popcount((R >> 1) & s) & 1)]), b[s], x[R], 0, 0, 0);
}

__device__ __forceinline__ uint32_t f16_pair(float x, float y) {
  const f16x2 h = {(_Float16)x, (_Float16)y};
  return __builtin_bit_cast(uint32_t, h);
}
__device__ __forceinline__ f16x8 operand(uint32_t a, uint32_t b, uint32_t c, uint32_t d) { return __builtin_bit_cast(f16x8, u32x4{a, b, c, d}); }
// x as one fp16 number (TERMS = 1), or as the sum of two: the second is what the first leaves, of that very first number.  (The compiler would round x twice,
// once from the product that x comes from and once from x, and the two may be neighbours: scores of such rows were off by 2^-13 of a coordinate.)
template <int TERMS> __device__ __forceinline__ void split_f16(const float (&x)[8], f16x8 (&out)[TERMS]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = f16_pair(x[2 * i], x[2 * i + 1]);
  if constexpr (TERMS == 2) {
    uint32_t rest[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      asm("" : "+v"(w[i]));
      const f16x2 h = __builtin_bit_cast(f16x2, w[i]);
      rest[i] = f16_pair(x[2 * i] - (float)h[0], x[2 * i + 1] - (float)h[1]);
    }
    out[1] = operand(rest[0], rest[1], rest[2], rest[3]);
  }
  out[0] = operand(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ f32x4 mfma(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// ---------------------------------------------------------------- codes
template <int NCW, int TERMS> struct Codes {
  static constexpr bool kRtn = is_rtn(NCW);
  static constexpr int c = CodeBits<NCW>::c;               // bits per pair of values
  static constexpr int kRow = kGroup / 2 * c / 8;          // bytes of a token's codes in one head
  // The grid in LDS: a row of 256 bytes per point that holds it over and over (fp16 pair, or that and the rest of it), so that every
  // lane finds its own copy in its own banks, and the byte offset of a look-up is (code << 8 | the lane's copy), put together by one byte permute.
  static constexpr int kTableBytes = kRtn ? 0 : NCW * 256;
  static constexpr int kEntry = 4 * TERMS;
  static constexpr int kScaleBytes = kRtn ? 512 : 128;     // per wave
  
  // A lane's points, kPoints l ... (fewer points than lanes: l modulo the points), on their way to LDS.
  static constexpr int kPoints = NCW / 64 > 0 ? NCW / 64 : 1;
  struct Points { float x[2 * kPoints]; };
  static __device__ __forceinline__ Points request_points(const float* __restrict__ codebook, int lane) {
    Points p = {};
    if constexpr (!kRtn) __builtin_memcpy(&p, codebook + 2 * kPoints * (lane & (NCW / kPoints - 1)), sizeof(p));
    return p;
  }
  // The grid's exponent e, so that it is held times 2^-e.
  static __device__ __forceinline__ int exponent(const Points& p) {
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < 2 * kPoints; ++i) top = fmaxf(top, fabsf(p.x[i]));
    top = column_max(top);
    top = fmaxf(top, row_xor8(top));
    top = fmaxf(top, octet_mirror(top));
    top = fmaxf(top, quad_xor<1>(top));
    top = fmaxf(top, quad_xor<2>(top));
    return max(uniform(__builtin_amdgcn_frexp_expf(top)), -100);
  }
  // -> exponent e of the grid.  Wave `wave` of WAVES writes its share of every point's row; lanes start at different
  // places of their rows, so that their banks differ.
  template <int WAVES> static __device__ __forceinline__ int stage(const Points& p, unsigned char* lds, int lane, int wave) {
    if constexpr (kRtn) return 0;
    const int e = exponent(p);
    constexpr int kLanes = NCW / kPoints;                  // lanes that hold different points
    constexpr int kChunks = 16 * kLanes / 64;              // 16-byte pieces of its points' rows that a lane of the workgroup writes, over the waves
#pragma unroll
    for (int i = 0; i < kPoints; ++i) {
      const float x = __builtin_ldexpf(p.x[2 * i], -e), y = __builtin_ldexpf(p.x[2 * i + 1], -e);
      uint32_t hi = f16_pair(x, y);
      uint32_t other = hi;
      if constexpr (TERMS == 2) {
        asm("" : "+v"(hi));                                // (as in split_f16)
        const f16x2 h = __builtin_bit_cast(f16x2, hi);
        other = f16_pair(x - (float)h[0], y - (float)h[1]);
      }
      const int point = kPoints * (lane & (kLanes - 1)) + i, turn = lane / kLanes;
#pragma unroll
      for (int k = 0; k < (kChunks + WAVES - 1) / WAVES; ++k) {
        const int chunk = turn + (64 / kLanes) * (wave + WAVES * k);
        if (kChunks % WAVES == 0 || wave + WAVES * k < kChunks)
          *reinterpret_cast<u32x4*>(lds + 256 * point + 16 * ((chunk + lane) & 15)) = u32x4{hi, other, hi, other};
      }
    }
    return e;
  }

  // ---- the row's query: lane group g holds coordinates 32 g ..., uniform: 16 g ... of both halves
  template <typename T> struct Query { u32x4 w[2 * sizeof(T)], signs[kRtn ? 1 : 2]; };      // as loaded
  template <typename T> static __device__ __forceinline__ Query<T> request_query(const T* __restrict__ row, const int8_t* signs, int h, int g) {
    Query<T> q;
    constexpr int kHalf = sizeof(T);                       // 16-byte words of 16 values
#pragma unroll
    for (int i = 0; i < 2 * kHalf; ++i)
      q.w[i] = reinterpret_cast<const u32x4*>(row + (kRtn ? 64 * (i / kHalf) + 16 * g : 32 * g + 16 * (i / kHalf)))[i % kHalf];
    if constexpr (!kRtn) {
#pragma unroll
      for (int i = 0; i < 2; ++i) q.signs[i] = reinterpret_cast<const u32x4*>(signs + h * kGroup + 32 * g)[i];
    }
    return q;
  }
  // ... rotated (grids; without the factor 1 / sqrt(128))
  static __device__ __forceinline__ uint32_t sign_bit(const u32x4 (&signs)[kRtn ? 1 : 2], int r) {      // bit 31: the sign of coordinate r of the lane's
    return (signs[r >> 4][(r >> 2) & 3] << (24 - 8 * (r & 3))) & 0x80000000u;
  }
  template <typename T> static __device__ __forceinline__ void rotate_query(const Query<T>& q, int lane, float (&v)[32]) {
    if constexpr (sizeof(T) == 2 && !kRtn) {
      bf16x8 b[4];
      f32x4 x[8] = {};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        u32x4 w = q.w[i];
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] ^= sign_bit(q.signs, 8 * i + 2 * k) >> 16 | sign_bit(q.signs, 8 * i + 2 * k + 1);
        b[i] = __builtin_bit_cast(bf16x8, w);
      }
      hadamard_columns(b, x, lane);
#pragma unroll
      for (int r = 0; r < 32; ++r) v[r] = x[r >> 2][r & 3];
      return;
    }
#pragma unroll
    for (int i = 0; i < 2 * (int)sizeof(T); ++i) {
      if constexpr (sizeof(T) == 2) {
        unpack_bf16x8(q.w[i], &v[8 * i]);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[4 * i + k] = __uint_as_float(q.w[i][k]);
      }
    }
    if constexpr (!kRtn) {
#pragma unroll
      for (int r = 0; r < 32; ++r) v[r] = __uint_as_float(__float_as_uint(v[r]) ^ sign_bit(q.signs, r));
      wht_columns(v);
    }
  }
  static __device__ __forceinline__ void pack_query(const float (&v)[32], f16x8 (&q)[TERMS][4], float (&qsum)[2]) {
    qsum[0] = qsum[1] = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = v[8 * j + i];
      f16x8 part[TERMS];
      split_f16<TERMS>(x, part);
#pragma unroll
      for (int n = 0; n < TERMS; ++n) {
        if constexpr (!kRtn) {
          q[n][j] = part[n];
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) qsum[j >> 1] += (float)part[n][i];
        }
      }
      if constexpr (kRtn) {
#pragma unroll
        for (int n = 0; n < TERMS; ++n) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            // value 8 (j & 1) + i of the half's 16: where its code comes up, and by how much it is too large there
            const int r = 8 * (j & 1) + i;
            const int to_j = NCW == kRtn4 ? j : 2 * (j >> 1) + ((r >> 2) & 1);
            const int at = NCW == kRtn4 ? 2 * (i & 3) + (i >> 2) : 2 * (r & 3) + (r >> 3);
            q[n][to_j][at] = part[n][i] * (_Float16)(1.0f / (float)field_scale(NCW == kRtn4 ? i & 1 : r & 3));
          }
        }
      }
    }
    if constexpr (kRtn) {
      qsum[0] = __builtin_ldexpf(column_sum(qsum[0]), -kFieldExp);
      qsum[1] = __builtin_ldexpf(column_sum(qsum[1]), -kFieldExp);
    }
  }
  // uniform: the k-th field of a half-word is masked in place, and so this many times its code
  static constexpr int field_scale(int k) { return 1 << (NCW * k); }
  static constexpr uint32_t field_mask(int k) { return 0x00010001u * (((1u << NCW) - 1u) << (NCW * k)); }
  // ... as fp16 numbers.  One term: the bits as they are, a subnormal number, times 2^-kFieldExp.  Two terms: a normal number, by way of 1024 + it (the
  // matrix instructions align products by their exponents before they add them, and a subnormal number's is 10 above its bits: sums kept about 2^-17).
  static constexpr int kFieldExp = TERMS == 1 ? 24 : 0;
  static __device__ __forceinline__ uint32_t small_ints(uint32_t x) {
    if constexpr (TERMS == 1) return x;
    const f16x2 k = {(_Float16)1024.0f, (_Float16)1024.0f};
    return __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, x | 0x64006400u) - k);
  }
  static __device__ __forceinline__ uint32_t field(uint32_t x, int k) { return small_ints(x & field_mask(k)); }
  static constexpr int kFields = NCW == kRtn4 ? 2 : 4;     // fields of a byte

  // ---- a tile's codes and scales on their way: keys of tokens 8 (m / 4) + m % 4 (+ 4), the lane group's share of the coordinates;
  // values of tokens 8 g ..., 8 coordinates; the scale word of token lane % 32, lanes from 32 on: of the values
  struct Keys {
    u32x4 k[2];
    std::conditional_t<kRtn, u32x2, uint32_t> scale;
  };
  struct Values { uint32_t v[8]; };
  // FAR: an array of the pool is larger than 4 GiB.  Otherwise a lane's place is a 32-bit offset from addresses that are the same for all lanes
  // (the pool's, and those of its second to eighth row), which takes no vector instruction but the choice of its group's row.
  template <bool FAR> struct Place {
    const uint8_t* base;
    std::conditional_t<FAR, uint64_t, uint32_t> at;
    __device__ __forceinline__ Place(const void* pool, const Rows& rows, int j, uint32_t row_bytes, uint32_t lane_at) : base(static_cast<const uint8_t*>(pool)) {
      if constexpr (FAR) {
        at = (uint64_t)row_of(rows, j) * row_bytes + lane_at;
      } else {
        Rows bytes;
#pragma unroll
        for (int i = 0; i < 4; ++i) bytes.r[i] = (int)((uint32_t)max(rows.r[i], 0) * row_bytes);
        at = (uint32_t)pick_of(bytes, j) + lane_at;
      }
    }
    template <typename W> __device__ __forceinline__ W load(uint32_t more) const {       // `more`: the same for all lanes
      uint64_t from = reinterpret_cast<uint64_t>(base) + more;
      asm("" : "+s"(from));                                // (a sum in scalar registers, not one per lane)
      W w;
      __builtin_memcpy(&w, reinterpret_cast<const __attribute__((address_space(1))) uint8_t*>(from) + at, sizeof(W));
      return w;
    }
  };
  template <bool FAR, bool VALUES = true> static __device__ __forceinline__ Keys request_keys(const PagedAttendArgs& a, const Rows& rows, int h, int lane) {
    const int m = lane & 15, g = lane >> 4;
    const uint32_t row_bytes = (uint32_t)a.H * kRow, head = (uint32_t)h * kRow;
    Keys w;
    const Place<FAR> k(a.pool.k_codes, rows, m >> 2, row_bytes, (m & 3) * row_bytes + (kRtn ? c : 2 * c) * g);
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const uint32_t more = head + 4 * p * row_bytes;
      if constexpr (NCW == kRtn4) {
        const u32x2 x = k.template load<u32x2>(more), y = k.template load<u32x2>(more + 32);
        w.k[p] = u32x4{x.x, x.y, y.x, y.y};
      } else if constexpr (NCW == kRtn2) {
        w.k[p] = u32x4{k.template load<uint32_t>(more), k.template load<uint32_t>(more + 16), 0, 0};
      } else if constexpr (c == 8) {
        w.k[p] = k.template load<u32x4>(more);
      } else if constexpr (c == 4) {
        const u32x2 x = k.template load<u32x2>(more);
        w.k[p] = u32x4{x.x, x.y, 0, 0};
      } else {
        struct Three { uint32_t x, y, z; };
        const Three x = k.template load<Three>(more);
        w.k[p] = u32x4{x.x, x.y, x.z, 0};
      }
    }
    const uint16_t* const scales = !VALUES || lane < 32 ? a.pool.k_scales : a.pool.v_scales;
    const uint64_t at = (uint64_t)(row_of(rows, (lane >> 3) & 3) + (lane & 7)) * a.H + h;
    if constexpr (kRtn) w.scale = reinterpret_cast<const u32x2*>(scales)[at];
    else w.scale = scales[at];
    return w;
  }
  template <bool FAR> static __device__ __forceinline__ Values request_values(const PagedAttendArgs& a, const Rows& rows, int h, int lane) {
    const int m = lane & 15, g = lane >> 4;
    const uint32_t row_bytes = (uint32_t)a.H * kRow, head = (uint32_t)h * kRow;
    Values w;
    const Place<FAR> v(a.pool.v_codes, rows, g, row_bytes, c == 8 ? 4 * m : c == 4 ? 2 * m : max(3 * m - 1, 0));
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t more = head + e * row_bytes;
      if constexpr (c == 4) w.v[e] = v.template load<uint16_t>(more);
      else w.v[e] = v.template load<uint32_t>(more);       // (6 bits: the lane's 3 bytes, and the one before them)
    }
    return w;
  }

  // ---- scales: every lane's eight tokens 8 g ..., through LDS
  static __device__ __forceinline__ void put_scales(const Keys& w, unsigned char* lds, int lane) {
    uint16_t* const to = reinterpret_cast<uint16_t*>(lds);
    if constexpr (kRtn) {                                  // keys, values: step and zero point of the lower half, of the upper half
      uint16_t* const mine = to + (lane >> 5) * 128 + (lane & 31);
      mine[0] = (uint16_t)w.scale.x; mine[32] = (uint16_t)(w.scale.x >> 16);
      mine[64] = (uint16_t)w.scale.y; mine[96] = (uint16_t)(w.scale.y >> 16);
    } else {
      to[lane] = (uint16_t)w.scale;
    }
  }
  static constexpr int kKeys = 0, kValues = kRtn ? 4 : 1;  // rows of 32 half-words
  static __device__ __forceinline__ u32x4 eight(const unsigned char* lds, int row, int g) { return *reinterpret_cast<const u32x4*>(lds + 64 * row + 16 * g); }
  static __device__ __forceinline__ float half_at(const u32x4& w, int e) {
    const f16x8 h = __builtin_bit_cast(f16x8, w);
    return (float)h[e];
  }
  static __device__ __forceinline__ float int_at(const u32x4& w, int e) { return (float)((w[e >> 1] >> (16 * (e & 1))) & 0xffffu); }
  // the values' scales of the lane's tokens, per half (kHalves), and their zero points: fp16 numbers (times 2^-kFieldExp).  `there`: those from it on are 0
  static constexpr int kHalves = kRtn ? 2 : 1;
  static __device__ __forceinline__ u32x4 value_scales(const unsigned char* lds, int k, int g) { return eight(lds, kValues + 2 * k, g); }
  // BOUNDED: those that are none (beyond 1023, of tokens whose rows hold anything) are made finite, as their weight of 0 asks for
  template <bool BOUNDED> static __device__ __forceinline__ f16x8 zero_points(const unsigned char* lds, int k, int g, int there) {
    u32x4 w = eight(lds, kValues + 2 * k + 1, g);
    if (there < 8) SeenOf<false>{there}.keep(w);
    if constexpr (BOUNDED) w &= 0x03ff03ffu;
    return operand(small_ints(w.x), small_ints(w.y), small_ints(w.z), small_ints(w.w));
  }
  // power of two of the largest scale of the lane's tokens (at least the smallest fp16 number's)
  static __device__ __forceinline__ float lift_of(const u32x4 (&vs)[kHalves]) {
    const auto pair = [&](int k, int i) {
      const uint32_t w = vs[k][i];                         // (a cast of the element itself would take the vector's first)
      return __builtin_bit_cast(f16x2, w);
    };
    f16x2 top = pair(0, 0);
#pragma unroll
    for (int k = 0; k < kHalves; ++k)
#pragma unroll
      for (int i = k == 0 ? 1 : 0; i < 4; ++i) top = __builtin_elementwise_max(top, pair(k, i));
    return __builtin_amdgcn_logf(fmaxf(fmaxf((float)top[0], (float)top[1]), 0x1p-24f));
  }

  // ---- look-ups
  template <int TERM = 0> static __device__ __forceinline__ uint32_t point(const unsigned char* lds, uint32_t offset) {
    return *reinterpret_cast<const uint32_t*>(lds + offset + 4 * TERM);
  }
  // offset of the lane's copy (lane_at: 0 ... 255) of the point whose code is byte `k` of w
  static __device__ __forceinline__ uint32_t offset_of_byte(uint32_t w, int k, uint32_t lane_at) {
    return __builtin_amdgcn_perm(w, lane_at, 0x0c0c0400u + ((uint32_t)k << 8));
  }
  static __device__ __forceinline__ uint32_t lane_copy(int lane) { return (uint32_t)(lane * kEntry) & 255u; }
  // code i (compile time) of the packed codes in w
  template <int N> static __device__ __forceinline__ uint32_t offset(const uint32_t (&w)[N], int i, uint32_t lane_at) {
    if constexpr (c == 8) {
      return offset_of_byte(w[i >> 2], i & 3, lane_at);
    } else if constexpr (c == 4) {
      uint32_t x = (i & 1) ? w[i >> 3] >> 4 : w[i >> 3];
      x &= 0x0f0f0f0fu;
      return offset_of_byte(x, (i >> 1) & 3, lane_at);
    } else {
      const int bit = 6 * i, n = bit >> 5, sh = bit & 31;
      uint32_t x = w[n] >> sh;
      if (sh > 26) x |= w[n + 1 < N ? n + 1 : n] << (32 - sh);
      return (x & 63u) << 8 | lane_at;
    }
  }

  // What a lane keeps of one of its (one or two) rows.
  struct Column {
    f16x8 q[TERMS][4];
    float qsum[2];                                         // uniform: sum of the row's (rounded) query over each half
    float f;                                               // score in powers of two = f * sigma * sum
    int limit;                                             // last token that the row sees
    f32x4 o[8];
    f32x4 oz[kRtn ? 2 : 1];                                // uniform: sums of the zero points, per half
    float ref, sum;                                        // weights are 2^(score - ref)
  };
  // ---- scores of product p: s[column][half][p] += keys * query
  template <int COLS> static __device__ __forceinline__ void scores(const Keys& w, int p, const unsigned char* lds, int lane, const Column (&col)[COLS],
                                                                    f32x4 (&s)[COLS][kRtn ? 2 : 1][2]) {
    const uint32_t x[4] = {w.k[p].x, w.k[p].y, w.k[p].z, w.k[p].w};
    if constexpr (kRtn) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t y[4];
        const uint32_t d = NCW == kRtn4 ? x[j] : (j & 1) ? x[j >> 1] >> 8 : x[j >> 1];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = NCW == kRtn4 ? field((i & 2) ? d >> 8 : d, i & 1) : field(d, i);
        const f16x8 k = operand(y[0], y[1], y[2], y[3]);
#pragma unroll
        for (int n = 0; n < TERMS; ++n)
#pragma unroll
          for (int i = 0; i < COLS; ++i) s[i][j >> 1][p] = mfma(k, col[i].q[n][j], s[i][j >> 1][p]);
      }
    } else {
      const uint32_t at = lane_copy(lane);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = offset(x, 4 * j + i, at);
        const f16x8 k = operand(point(lds, o[0]), point(lds, o[1]), point(lds, o[2]), point(lds, o[3]));
#pragma unroll
        for (int i = 0; i < COLS; ++i) s[i][0][p] = mfma(k, col[i].q[0][j], s[i][0][p]);
        if constexpr (TERMS == 2) {
          const f16x8 rest = operand(point<1>(lds, o[0]), point<1>(lds, o[1]), point<1>(lds, o[2]), point<1>(lds, o[3]));
#pragma unroll
          for (int i = 0; i < COLS; ++i) {
            s[i][0][p] = mfma(k, col[i].q[1][j], s[i][0][p]);
            s[i][0][p] = mfma(rest, col[i].q[0][j], s[i][0][p]);
          }
        }
      }
    }
  }
  // ... of the lane's eight tokens, times the scales
  static __device__ __forceinline__ void scaled(const f32x4 (&s)[kRtn ? 2 : 1][2], const unsigned char* lds, int g, const float (&qsum)[2], float (&y)[8]) {
    const u32x4 ks = eight(lds, kKeys, g);
    if constexpr (kRtn) {
      const u32x4 kz = eight(lds, kKeys + 1, g), ks1 = eight(lds, kKeys + 2, g), kz1 = eight(lds, kKeys + 3, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float lo = __fmaf_rn(-int_at(kz, e), qsum[0], s[0][e >> 2][e & 3]), hi = __fmaf_rn(-int_at(kz1, e), qsum[1], s[1][e >> 2][e & 3]);
        y[e] = __fmaf_rn(lo, half_at(ks, e), hi * half_at(ks1, e));
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = s[0][e >> 2][e & 3] * half_at(ks, e);
    }
  }

  // ---- o[j] += values (coordinates: result()) * weights p * scale.  `there` of the lane's tokens are; masked: a row sees the first seen[] of them, and what the
  // scales of the others are is no matter (0 times a number that is not finite would be): with one row a lane they are 0 already, with two the weights become 0.
  template <int COLS, typename Seen> static __device__ __forceinline__ void values(const Values& w, const unsigned char* scales, int there, bool masked, const Seen (&seen)[COLS],
                                                                    const float (&p)[COLS][8], const u32x4 (&vs)[kHalves], const unsigned char* lds, int lane,
                                                                    Column (&col)[COLS]) {
    f16x8 b[COLS][kHalves][TERMS];
#pragma unroll
    for (int n = 0; n < COLS; ++n)
#pragma unroll
      for (int k = 0; k < kHalves; ++k) {
        float weight[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) weight[e] = p[n][e] * half_at(vs[k], e);
        split_f16<TERMS>(weight, b[n][k]);
      }
    if (COLS > 1 && masked) {
      asm volatile("");
#pragma unroll
      for (int n = 0; n < COLS; ++n)
#pragma unroll
        for (int k = 0; k < kHalves; ++k)
#pragma unroll
          for (int i = 0; i < TERMS; ++i) {
            u32x4 x = __builtin_bit_cast(u32x4, b[n][k][i]);
            seen[n].keep(x);
            b[n][k][i] = __builtin_bit_cast(f16x8, x);
          }
    }
    if constexpr (kRtn) {
      // All rows of an operand have to be of one half (the weights are the half's): of the eight codes that a lane holds, lanes m and m ^ 8
      // exchange four.  Lower half-word: coordinates of the lower half, upper one: of the upper half.
      uint32_t d[8];
      const uint32_t pick = c == 8 ? ((lane & 8) ? 0x07060302u : 0x01000504u) : ((lane & 8) ? 0x0c050c01u : 0x0c000c04u);
#pragma unroll
      for (int e = 0; e < 8; ++e) d[e] = __builtin_amdgcn_perm(w.v[e], __float_as_uint(row_xor8(__uint_as_float(w.v[e]))), pick);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const f16x8 z = zero_points<std::is_same<Seen, SeenOf<true>>::value>(scales, k, lane >> 4, there);
#pragma unroll
        for (int i = 0; i < COLS; ++i)
#pragma unroll
          for (int n = 0; n < TERMS; ++n) col[i].oz[k] = mfma(z, b[i][k][n], col[i].oz[k]);
#pragma unroll
        for (int byte = 0; byte < 4 / kFields; ++byte) {
          uint32_t x[4];                                   // tokens 2 i and 2 i + 1 in the halves
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] = __builtin_amdgcn_perm(d[2 * i + 1], d[2 * i], 0x0c040c00u + 0x00010001u * (2 * k + byte));
#pragma unroll
          for (int f = 0; f < kFields; ++f) {
            const f16x8 v = operand(field(x[0], f), field(x[1], f), field(x[2], f), field(x[3], f));
            const int j = 4 * k + kFields * byte + f;
#pragma unroll
            for (int i = 0; i < COLS; ++i)
#pragma unroll
              for (int n = 0; n < TERMS; ++n) col[i].o[j] = mfma(v, b[i][k][n], col[i].o[j]);
          }
        }
      }
    } else {
      const uint32_t at = lane_copy(lane), m = lane & 15;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t d[TERMS][8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t x[1] = {c == 6 ? w.v[e] >> (m != 0 ? 8 : 0) : w.v[e]};
          const uint32_t off = offset(x, i, at);
          d[0][e] = point(lds, off);
          if constexpr (TERMS == 2) d[1][e] = point<1>(lds, off);
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {                      // coordinates 2 i, 2 i + 1 of the lane's eight
          f16x8 v[TERMS];
#pragma unroll
          for (int n = 0; n < TERMS; ++n) {
            uint32_t x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = __builtin_amdgcn_perm(d[n][2 * e + 1], d[n][2 * e], k == 0 ? 0x05040100u : 0x07060302u);
            v[n] = operand(x[0], x[1], x[2], x[3]);
          }
#pragma unroll
          for (int n = 0; n < COLS; ++n) {
            f32x4& o = col[n].o[2 * i + k];
            o = mfma(v[0], b[n][0][0], o);
            if constexpr (TERMS == 2) {
              o = mfma(v[0], b[n][0][1], o);
              o = mfma(v[1], b[n][0][0], o);
            }
          }
        }
      }
    }
  }
  // the lane's 32 coordinates, in fours from coordinate(g, 4 i'): product j's row 4 g + i is coordinate 8 (4 g + i) + j, or (uniform) 8 ((4 g + i) % 8) +
  // 4 (g / 2) + j % 4 of half j / 4
  static __device__ __forceinline__ int coordinate(int g, int r) {
    return kRtn ? 64 * (r >> 4) + 8 * ((4 * g + ((r >> 2) & 3)) & 7) + 4 * (g >> 1) : 32 * g + r;
  }
  static __device__ __forceinline__ void result(const Column& col, int e, float (&v)[32]) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (kRtn) v[16 * (j >> 2) + 4 * i + (j & 3)] = __builtin_ldexpf(col.o[j][i] * (1.0f / (float)field_scale(j % kFields)) - col.oz[j >> 2][i], e);
        else v[8 * i + j] = __builtin_ldexpf(col.o[j][i], e);
      }
  }
};

// The lane's 32 coordinates of a row's result -> out.
template <typename T, int NCW> __device__ __forceinline__ void finish(const PagedAttendArgs& a, float (&v)[32], float sum, int h, int lane,
                                                                      bool there, int64_t row, int qh) {
  constexpr bool kRtn = is_rtn(NCW);
  float by = sum == 0.f ? 0.f : 1.0f / sum;                // (no token: 0)
  if constexpr (!kRtn) by *= kRsqrtG;
#pragma unroll
  for (int r = 0; r < 32; ++r) v[r] *= by;
  if constexpr (!kRtn && sizeof(T) == 2) {                 // (as two bf16 numbers: 2^-17 of a value, far below the rounding of the result)
    f32x4 x[8] = {};
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      bf16x8 b[4];
#pragma unroll
      for (int r = 0; r < 32; ++r) {
        const bf16_t part = static_cast<bf16_t>(v[r]);
        b[r >> 3][r & 7] = part;
        v[r] -= static_cast<float>(part);
      }
      hadamard_columns(b, x, lane);
    }
#pragma unroll
    for (int r = 0; r < 32; ++r) v[r] = x[r >> 2][r & 3];
  } else if constexpr (!kRtn) {
    wht_columns(v);
  }
  if constexpr (!kRtn) {
    float sf[32];
    load_signs(a.signs_v, h, lane >> 4, sf);
#pragma unroll
    for (int r = 0; r < 32; ++r) v[r] *= sf[r];
  }
  if (!there) return;
  T* const out = static_cast<T*>(a.out) + (row * a.q_heads + qh) * kGroup;
#pragma unroll
  for (int r = 0; r < 32; r += 4) {
    T* const at = out + Codes<NCW, 1>::coordinate(lane >> 4, r);
    if constexpr (sizeof(T) == 2) {
      *reinterpret_cast<u32x2*>(at) = u32x2{Storage<T>::pack2(v[r], v[r + 1]), Storage<T>::pack2(v[r + 2], v[r + 3])};
    } else {
      *reinterpret_cast<f32x4*>(at) = f32x4{v[r], v[r + 1], v[r + 2], v[r + 3]};
    }
  }
}

}  // namespace paged
}  // namespace aquakv
