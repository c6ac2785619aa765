// Attention of many queries over pages of codes (a chunk of a prompt behind what is cached): bf16 layers.  The kernel, which paged_tiles.hip and, for trees of drafted tokens, paged_tree.hip build.
//
// A workgroup of 8 waves takes 32 rows (query x query head) a wave of one kv head and walks the tokens in tiles of 64.  The waves turn a tile's
// codes into fp16 once, for all of them, keys [token][coordinate] and values [coordinate][token] in LDS (two buffers: the next tile is
// written while this one is multiplied), and multiply with 32x32x16 matrix instructions: S^T = K Q^T, O^T += V^T P.  As in paged_attend.hip the lane
// that gets scores holds them as the second product wants its operand: V's columns are in that order.
#pragma once
#include "paged_attend.h"

namespace aquakv {
namespace paged {

typedef float f32x16 __attribute__((ext_vector_type(16)));
constexpr int kTokens = 64;                                // of a tile
constexpr int kKeyBytes = kTokens * kGroup * 2;             // (values: as many)

// Coordinate (of 128) that row i of a 32-row operand R stands for, so that register n of lanes 32 hf ... of product R is coordinate
// 16 (2 R + n / 8) + 8 hf + n % 8: what such a lane holds of a vector as the other operand.  (Swaps bits 2 and 3.)
__device__ __forceinline__ int swapped(int d) { return (d & ~12) | (d & 4) << 1 | (d & 8) >> 1; }

// LDS places: 16-byte pieces of a row are shuffled so that the lanes that read one piece of 16 rows (keys), or of 8 pairs of rows (values), use
// different banks.
__device__ __forceinline__ uint32_t key_place(int token, int piece) { return 256 * token + 16 * (piece ^ (token & 15)); }
__device__ __forceinline__ uint32_t value_place(int row, int piece) { return 128 * row + 16 * (piece ^ ((row >> 1) & 7)); }

// x += H b, columns of 128 bf16 numbers on two lanes (b[s]: coordinates 16 s + 8 hf ...)
__device__ __forceinline__ void hadamard_pairs(const bf16x8 (&b)[8], f32x16 (&x)[4], int lane) {
  const uint32_t r = lane & 31, hf = lane >> 5, flip = 0x80008000u;
  const uint32_t p = 0x3f803f80u ^ ((r & 1) << 31) ^ (((r >> 2) & hf) ? flip : 0u), q = p ^ ((r & 2) ? flip : 0u);
  const uint32_t p2 = p ^ ((r & 8) ? flip : 0u), q2 = q ^ ((r & 8) ? flip : 0u), odd = (r & 16) ? flip : 0u;
  const u32x4 even = {p, q, p2, q2}, row[4] = {even, even ^ odd, even ^ flip, even ^ odd ^ flip};
#pragma unroll
  for (int s = 0; s < 8; ++s)
#pragma unroll
    for (int R = 0; R < 4; ++R)
      x[R] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, row[(s & 1) + 2 * (__builtin_popcount((s >> 1) & R) & 1)]), b[s], x[R], 0, 0, 0);
}
__device__ __forceinline__ float pair_max(float x) {       // over lanes l, l ^ 32
  float y = x;
  swap_lanes<32>(x, y);
  return fmaxf(x, y);
}

// ---------------------------------------------------------------- codes of a tile
// Wave `part` of the eight that a tile is shared out to: keys of tokens 8 part ... (a lane: 16 coordinates of a token), values of the eight tokens
// that operand piece `part` holds, 16 (part / 2) + 4 (part % 2) + {0 ... 3, 8 ... 11} (a lane: 2 coordinates).
// Operands are grid points, or (uniform) code - zero point, exact; scales stay fp32, a uniform row's one for each half of the coordinates.
template <int NCW, bool TREE> struct TileCodes {
  typedef Codes<NCW, 1> C;
  static constexpr bool kRtn = C::kRtn;
  // behind keys and values, fp32: scales of the keys, of the values (rows of kTokens; uniform: lower half, upper half), the largest of each eight of the
  // values', pages that are not there
  static constexpr int kHalves = C::kHalves, kLargest = 2 * kHalves * kTokens, kMissing = kLargest + 8, kBufferBytes = 2 * kKeyBytes + (kMissing + 8) * 4;
  static constexpr int c = C::c, kRow = C::kRow;
  u32x2 k;
  uint32_t v[8];
  u32x2 ks;                                                // the lane's token's scale word(s)
  uint32_t vs[kRtn ? 8 : 1];                               // grids: scale of token lane % 8 of the piece; uniform: of each, the lane's half
  bool missing;                                            // the keys' page is not in the pool
  int there[2];                                            // so many of the piece's first, second four tokens are there (the others hold anything)
  static __device__ __forceinline__ int value_token(int part, int e) { return 16 * (part >> 1) + 4 * (part & 1) + (e & 3) + 8 * (e >> 2); }

  __device__ __forceinline__ void request(const PagedAttendArgs& a, int b, int len, int h, int t, int part, int lane) {
    const uint32_t row_bytes = (uint32_t)a.H * kRow;
    const int key_group_row = group_row(a, b, t / 8 + part);
    const uint64_t key_row = (uint64_t)max(key_group_row, 0);
    missing = key_group_row < 0;
    const int group[2] = {group_row(a, b, t / 8 + (part & ~1)), group_row(a, b, t / 8 + (part | 1))};
    const uint64_t value_row[2] = {(uint64_t)max(group[0], 0) + 4 * (part & 1), (uint64_t)max(group[1], 0) + 4 * (part & 1)};
#pragma unroll
    for (int i = 0; i < 2; ++i) there[i] = group[i] < 0 ? 0 : len - (t + value_token(part, 4 * i));
    const uint8_t* const kp = a.pool.k_codes + (key_row * row_bytes + h * kRow) + (uint32_t)(lane >> 3) * row_bytes;
    if constexpr (c == 8) {
      k = *reinterpret_cast<const u32x2*>(kp + 8 * (lane & 7));
    } else if constexpr (c == 4) {
      k = u32x2{*reinterpret_cast<const uint32_t*>(kp + 4 * (lane & 7)), 0};
    } else {                                               // 6 bytes, from the second pieces on with the 2 before them
      __builtin_memcpy(&k, kp + max(6 * (lane & 7) - 2, 0), 8);
    }
    const uint64_t key_group = (key_row + (lane >> 3)) * a.H + h;
    if constexpr (kRtn) ks = reinterpret_cast<const u32x2*>(a.pool.k_scales)[key_group];
    else ks = u32x2{a.pool.k_scales[key_group], 0};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint64_t row = value_row[e >> 2] + (e & 3);
      const uint8_t* const vp = a.pool.v_codes + (row * row_bytes + h * kRow);
      if constexpr (c == 8) {
        v[e] = vp[lane];
      } else if constexpr (c == 4) {
        v[e] = vp[lane >> 1];
      } else {
        uint16_t two;
        __builtin_memcpy(&two, vp + min((6 * lane) >> 3, 46), 2);
        v[e] = two;
      }
      if constexpr (kRtn) vs[e] = reinterpret_cast<const uint32_t*>(a.pool.v_scales)[(row * a.H + h) * 2 + (lane >> 5)];
    }
    if constexpr (!kRtn) vs[0] = a.pool.v_scales[((lane & 4 ? value_row[1] : value_row[0]) + (lane & 3)) * a.H + h];
  }
  static __device__ __forceinline__ int group_row(const PagedAttendArgs& a, int b, uint32_t group) {
    uint32_t page = (uint32_t)(((uint64_t)group * a.page_magic) >> 32), in = group - page * a.page_groups;
    if (in >= a.page_groups) { ++page; in -= a.page_groups; }
    const int at = page < (uint32_t)a.table_pages ? const_ints(a.page_table)[(int64_t)b * a.table_pages + page] : -1;
    return (uint32_t)at < (uint32_t)a.pool.n_pages ? at * a.pool.page_tokens + (int)in * 8 : -1;
  }

  // a lane's keys and values to the buffer
  __device__ __forceinline__ void store(const unsigned char* table, unsigned char* buffer, int part, int lane) const {
    unsigned char* const values = buffer + kKeyBytes;
    float* const scales = reinterpret_cast<float*>(buffer + 2 * kKeyBytes);
    const int token = 8 * part + (lane >> 3), piece = 2 * (lane & 7);
    u32x4 out[2];
    if constexpr (kRtn) {
      const bool upper = (lane & 7) >= 4;
      const uint32_t word = upper ? ks.y : ks.x;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        out[i >> 2][i & 3] = NCW == kRtn4 ? less_zero<0>(i < 4 ? k.x : k.y, i & 3, word) : (i & 1) ? less_zero<2>(k.x, i >> 1, word) : less_zero<0>(k.x, i >> 1, word);
      if ((lane & 3) == 0) scales[(upper ? kTokens : 0) + token] = half_bits_to_float((uint16_t)word);
    } else {
      const uint32_t at = C::lane_copy(lane);
      const uint32_t w[2] = {c == 6 ? ((lane & 7) ? __builtin_amdgcn_alignbit(k.y, k.x, 16) : k.x) : k.x, c == 6 ? ((lane & 7) ? k.y >> 16 : k.y) : k.y};
#pragma unroll
      for (int i = 0; i < 8; ++i) out[i >> 2][i & 3] = C::point(table, C::offset(w, i, at));
      if ((lane & 7) == 0) scales[token] = half_bits_to_float((uint16_t)ks.x);
    }
    *reinterpret_cast<u32x4*>(buffer + key_place(token, piece)) = out[0];
    *reinterpret_cast<u32x4*>(buffer + key_place(token, piece + 1)) = out[1];
    // values: coordinates 2 lane, 2 lane + 1 of the piece's eight tokens.  (Their scales bound the weights: those of tokens that are not there are 0.)
    uint32_t d[8];
    float most = 0.f;
    if constexpr (kRtn) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        uint32_t word = (e & 3) < there[e >> 2] ? vs[e] : 0u;
        if constexpr (TREE) word &= 0x03ffffffu;           // (a draft that nobody sees may hold anything: its zero point has to be finite, as its weight of 0 asks for)
        const float step = half_bits_to_float((uint16_t)word);
        d[e] = less_zero<0>(NCW == kRtn4 ? v[e] : v[e] >> (4 * (lane & 1)), 0, word);
        most = fmaxf(most, step);
        if ((lane & 31) == 0) scales[(2 + (lane >> 5)) * kTokens + value_token(part, e)] = step;
      }
      most = pair_max(most);
    } else {
      const uint32_t at = C::lane_copy(lane);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t code = c == 8 ? v[e] : c == 4 ? (v[e] >> (4 * (lane & 1))) & 15u : (v[e] >> (6 * lane - 8 * min((6 * lane) >> 3, 46))) & 63u;
        d[e] = C::point(table, code << 8 | at);
      }
      most = (lane & 3) < (lane & 4 ? there[1] : there[0]) ? half_bits_to_float((uint16_t)vs[0]) : 0.f;
      if (lane < 8) scales[kHalves * kTokens + value_token(part, lane)] = most;
      most = fmaxf(most, quad_xor<1>(most));
      most = fmaxf(most, quad_xor<2>(most));
      most = fmaxf(most, octet_mirror(most));
    }
    if (lane == 0) {
      scales[kLargest + part] = most;
      scales[kMissing + part] = missing ? 1.0f : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t pick = i == 0 ? 0x05040100u : 0x07060302u;
      u32x4 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = __builtin_amdgcn_perm(d[2 * e + 1], d[2 * e], pick);
      *reinterpret_cast<u32x4*>(values + value_place(swapped(2 * lane + i), part)) = x;
    }
  }
  // uniform: fields F and F + 1 of byte `byte` of x, less the zero point in the upper half of `word`.  A field that is masked in place is 2^s times its code; behind
  // the bits of 1024 it is an fp16 number, 2^-s times which is 2^(10 - s) + code: one instruction takes that and the zero point off.  All of it is exact (zero
  // points up to 1023, as in the other kernel).
  template <int F> static __device__ __forceinline__ uint32_t less_zero(uint32_t x, int byte, uint32_t word) {
    constexpr uint32_t s0 = NCW * F, s1 = NCW * (F + 1), mask = (1u << NCW) - 1u;
    constexpr float by0 = 1.0f / (1 << s0), by1 = 1.0f / (1 << s1);
    constexpr f16x2 by = {(_Float16)by0, (_Float16)by1}, less = {(_Float16)(-1024.0f * by0), (_Float16)(-1024.0f * by1)};
    const uint32_t both = __builtin_amdgcn_perm(x, x, 0x0c000c00u + 0x00010001u * (uint32_t)byte);
    const uint32_t y = (both & (mask << s0 | mask << (16 + s1))) | 0x64006400u;
    const _Float16 zero = (_Float16)(uint16_t)(word >> 16);
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(__builtin_bit_cast(f16x2, y), by, less - f16x2{zero, zero}));
  }
};

// ---------------------------------------------------------------- the kernel
// 2048 queries of 32 heads over 12 288 tokens of 8 kv heads, 256 points: 503 to 523 us, 722 to 752 TFLOP/s (a library product of fp16 matrices of 8192 reaches 1319);
// 64 points 539, 16 points 511, uniform 4 bits 604, 2 bits 620 (weights and scores of each half).
// One workgroup a CU, two waves a SIMD (accumulators, query and a tile's codes in 236 to 248 registers): matrix cores busy in a third of the cycles, vector
// pipes in half of them; a wave's chain of products, maximum, exponentials and conversion is what is left, and the two waves of a SIMD do not hide it for each
// other.  Without the conversion of codes it would take 410 us, without the operands' LDS reads 465, without the exponentials 475.  Slower: 64 rows a
// wave (1010 us: accumulators moved between register files), waves in turns by barriers (703), operands requested ahead by hand (515, spills).
template <int NCW, bool TREE>
__global__ __launch_bounds__(64 * kTileWaves) __attribute__((amdgpu_waves_per_eu(2, 2))) void paged_tiles_kernel(const PagedAttendArgs a) {
  typedef Codes<NCW, 1> C;
  typedef TileCodes<NCW, TREE> Tile;
  constexpr bool kRtn = C::kRtn;
  constexpr int kHalves = Tile::kHalves, kBufferBytes = Tile::kBufferBytes;
  __shared__ __align__(256) unsigned char lds[C::kTableBytes + 2 * kBufferBytes];
  unsigned char* const buffers = lds + C::kTableBytes;
  const int lane = threadIdx.x & 63, col = lane & 31, hf = lane >> 5, wave = uniform(threadIdx.x >> 6);
  const typename C::Points points = C::request_points(a.codebook, lane);
  const int h = blockIdx.x % a.H;
  int piece, block, b, first_result, results;
  TokenRange range = {};
  if constexpr (TREE) {                                    // blockIdx: (piece of all sequences and kv head, block of rows)
    const int item = blockIdx.x / a.H;
    const Share share = share_of<kTokens, true>(a, lane, item);
    if (share.b < 0) return;
    b = share.b; piece = share.piece; block = blockIdx.y;
    first_result = share.results; results = share.pieces;      // (sequences in one piece keep none)
    range = {share.tiles, 0};
  } else {                                                 // (piece, block of rows: the last ones, which see most tokens, first; kv head), sequence
    piece = (blockIdx.x / a.H) % a.slots; block = a.row_blocks - 1 - blockIdx.x / a.H / a.slots; b = blockIdx.y;
    first_result = b * a.slots; results = a.slots;
  }
  const PagedQueries w = paged_queries(a, b);
  const int rep = a.q_heads / a.H, n_rows = w.n * rep, row0 = block * kTileRows;
  if (row0 >= n_rows) return;
  const int row = row0 + 32 * wave + col, qi = row / rep, qh = h * rep + row % rep;
  const bool row_there = row < n_rows;
  const int past = w.len - w.count;                        // tokens ahead of the queries' own
  const int limit = row_there ? past + qi : -1;
  const int wave_first = TREE ? past - 1 : uniform(past + min(row0 + 32 * wave, n_rows - 1) / rep);      // smallest limit of the wave's rows
  const int last_limit = TREE ? w.len - 1 : uniform(past + min(row0 + kTileRows - 1, n_rows - 1) / rep);
  range = piece_range(piece, TREE ? range.begin : (tiles_of_tokens(last_limit + 1, kTokens) + a.slots - 1) / a.slots, kTokens, last_limit + 1);
  const int t_begin = range.begin, t_end = range.end;

  Tile codes;
  const auto request = [&](int t) { codes.request(a, b, w.len, h, t, wave, lane); };
  const auto store = [&](int n) { codes.store(lds, buffers + n * kBufferBytes, wave, lane); };
  if (t_begin < t_end) request(t_begin);
  const int c_exp = C::template stage<kTileWaves>(points, lds, lane, wave);

  // ---- the rows' queries
  f16x8 q[8];
  float f;
  {
    const bf16_t* const src = static_cast<const bf16_t*>(a.q) + (w.first + (row_there ? qi : 0)) * a.q_stride + (row_there ? qh : h * rep) * kGroup + 8 * hf;
    float x[64];
    u32x4 raw[8];
#pragma unroll
    for (int s = 0; s < 8; ++s) raw[s] = *reinterpret_cast<const u32x4*>(src + 16 * s);
    if constexpr (!kRtn) {
      bf16x8 bq[8];
      const int8_t* const signs = a.signs_k + h * kGroup + 8 * hf;
#pragma unroll
      for (int s = 0; s < 8; ++s) {
        const u32x2 sg = *reinterpret_cast<const u32x2*>(signs + 16 * s);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t two = i < 2 ? sg.x >> (16 * i) : sg.y >> (16 * (i - 2));
          raw[s][i] ^= (two << 8 & 0x8000u) | (two << 16 & 0x80000000u);
        }
        bq[s] = __builtin_bit_cast(bf16x8, raw[s]);
      }
      f32x16 y[4] = {};
      hadamard_pairs(bq, y, lane);
#pragma unroll
      for (int r = 0; r < 64; ++r) x[r] = y[r >> 4][r & 15];
    } else {
#pragma unroll
      for (int s = 0; s < 8; ++s) unpack_bf16x8(raw[s], &x[8 * s]);
    }
    const float by = a.scale * 1.4426950408889634f * (kRtn ? 1.0f : kRsqrtG);
    float top = 0.f;
#pragma unroll
    for (int r = 0; r < 64; ++r) top = fmaxf(top, fabsf(x[r]));
    const int e = max(__builtin_amdgcn_frexp_expf(pair_max(top) * fabsf(by)), -100);
    f = __builtin_ldexpf(1.0f, min(e - kQueryExp + c_exp, 126));
    const float scaled = __builtin_ldexpf(by, kQueryExp - e);
#pragma unroll
    for (int s = 0; s < 8; ++s)
#pragma unroll
      for (int i = 0; i < 8; ++i) q[s][i] = (_Float16)(x[8 * s + i] * scaled);
  }
  __syncthreads();                                         // the grid's copies are there
  f32x16 o[4] = {};
  float ref = -3.0e38f, sum = 0.f;
  if (t_begin < t_end) store(0);
  __syncthreads();
  if (t_begin + kTokens < t_end) request(t_begin + kTokens);
  int n = 0;
#pragma unroll 1
  for (int t = t_begin; t < t_end; t += kTokens, n ^= 1) {
    const unsigned char* const buffer = buffers + n * kBufferBytes;
    const float* const scales = reinterpret_cast<const float*>(buffer + 2 * kKeyBytes);
    // groups of 8 tokens whose page is not in the pool
    const uint32_t missing = (uint32_t)__builtin_amdgcn_ballot_w64(scales[Tile::kMissing + (lane & 7)] != 0.f) & 255u;
    const bool masked = t + kTokens - 1 > wave_first || missing != 0;
    float lift;                                            // power of two of the tile's largest scale
    {
      const f32x4 x = *reinterpret_cast<const f32x4*>(scales + Tile::kLargest), y = *reinterpret_cast<const f32x4*>(scales + Tile::kLargest + 4);
      lift = __builtin_amdgcn_logf(fmaxf(fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3]))), 0x1p-24f));
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {                          // 32 tokens each
      f32x16 part[kHalves] = {};
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        f32x16& x = part[k * kHalves / 8];
        x = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const f16x8*>(buffer + key_place(32 * i + col, 2 * k + hf)), q[k], x, 0, 0, 0);
      }
      // the next tile's codes to the other buffer
      if (i == 0 && t + kTokens < t_end) {
        store(n ^ 1);
        if (t + 2 * kTokens < t_end) request(t + 2 * kTokens);
      }
      // register 4 j + e is token 32 i + 8 j + 4 hf + e
      f32x16& s = part[0];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float* const at = scales + 32 * i + 8 * j + 4 * hf;
        const f32x4 sk = *reinterpret_cast<const f32x4*>(at);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[4 * j + e] *= sk[e];
        if constexpr (kRtn) {
          const f32x4 upper = *reinterpret_cast<const f32x4*>(at + kTokens);
#pragma unroll
          for (int e = 0; e < 4; ++e) s[4 * j + e] = __fmaf_rn(part[1][4 * j + e], upper[e], s[4 * j + e]);
        }
      }
      // of tokens 32 i + 8 j + 4 hf ... the row sees so many
      const auto seen_of = [&](int j) {
        SeenOf<TREE> seen;
        const int from = t + 32 * i + 8 * j + 4 * hf;
        const bool there = !((missing >> (4 * i + j)) & 1);
        if constexpr (TREE) seen.bits = there && row_there ? tree_bits(a, w.first + qi, from - past) & first_bits(w.len - from) : 0u;
        else seen.n = there ? limit + 1 - from : 0;
        return seen;
      };
      const auto value_scales = [&](int half, int j) { return *reinterpret_cast<const f32x4*>(scales + (kHalves + half) * kTokens + 32 * i + 8 * j + 4 * hf); };
      float own_lift = lift;
      if (masked) {
        asm volatile("");                                  // (a branch: the selects would cost every tile an instruction and a half per score)
        float most = 0x1p-24f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const SeenOf<TREE> seen = seen_of(j);
#pragma unroll
          for (int e = 0; e < 4; ++e) s[4 * j + e] = seen.has(e) ? s[4 * j + e] : -INFINITY;
#pragma unroll
          for (int half = 0; half < kHalves; ++half) {
            const f32x4 sv = value_scales(half, j);
#pragma unroll
            for (int e = 0; e < 4; ++e) most = fmaxf(most, seen.has(e) ? sv[e] : 0.f);
          }
        }
        own_lift = __builtin_amdgcn_logf(most);
      }
      // the largest weight that the scores allow
      float top = s[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) top = fmaxf(top, s[r]);
      if (__builtin_amdgcn_ballot_w64(__fmaf_rn(top, f, own_lift - ref) > kTopExp) != 0) {
        const float moved = fmaxf(ref, pair_max(__fmaf_rn(top, f, own_lift)) - kStartExp);
        const float by = __builtin_amdgcn_exp2f(ref - moved);
        ref = moved;
        sum *= by;
#pragma unroll
        for (int R = 0; R < 4; ++R) o[R] *= by;
      }
      float p[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) p[r] = __builtin_amdgcn_exp2f(__fmaf_rn(s[r], f, -ref));
      sum += sum_of(p);
      const unsigned char* const values = buffer + kKeyBytes;
#pragma unroll
      for (int k = 0; k < 2; ++k) {                        // 16 tokens each
        f16x8 weight[kHalves];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
          for (int half = 0; half < kHalves; ++half) {
            const f32x4 sv = value_scales(half, 2 * k + j);
#pragma unroll
            for (int e = 0; e < 4; ++e) weight[half][4 * j + e] = (_Float16)(p[8 * k + 4 * j + e] * sv[e]);
          }
        }
        if (masked) {                                      // (a scale that is not finite, of a token that the row does not see, would make its weight NaN)
          asm volatile("");
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const SeenOf<TREE> seen = seen_of(2 * k + j);
#pragma unroll
            for (int half = 0; half < kHalves; ++half)
#pragma unroll
              for (int e = 0; e < 4; ++e) weight[half][4 * j + e] = seen.has(e) ? weight[half][4 * j + e] : (_Float16)0.f;
          }
        }
#pragma unroll
        for (int R = 0; R < 4; ++R)
          o[R] = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const f16x8*>(values + value_place(32 * R + col, 4 * i + 2 * k + hf)),
                                                        weight[R * kHalves / 4], o[R], 0, 0, 0);
      }
    }
    __syncthreads();
  }

  // ---- results: register n of product R is coordinate 16 (2 R + n / 8) + 8 hf + n % 8
  sum = far_sum<32>(sum);
  if (TREE && a.heads != nullptr && block == 0 && h == 0 && piece == 0 && threadIdx.x == 0) a.heads[b] = int2{first_result, results};
  if (results > 1) {
    if (!TREE && block == 0 && h == 0 && piece == 0 && threadIdx.x == 0) a.heads[b] = int2{first_result, results};
    if (!row_there) return;
    const int64_t at = ((int64_t)(first_result + piece) * a.max_queries + qi) * a.q_heads + qh;
    float* const part = a.part + at * kGroup + 8 * hf;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      f32x4 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = __builtin_ldexpf(o[r >> 2][4 * (r & 3) + e], c_exp);
      *reinterpret_cast<f32x4*>(part + 16 * (r >> 1) + 4 * (r & 1)) = x;
    }
    if (hf == 0) *reinterpret_cast<f32x2*>(a.stats + 2 * at) = f32x2{ref, sum};
    return;
  }
  const float by = sum == 0.f ? 0.f : __builtin_ldexpf((kRtn ? 1.0f : kRsqrtG) / sum, c_exp);
#pragma unroll
  for (int R = 0; R < 4; ++R) o[R] *= by;
  if constexpr (!kRtn) {
    f32x16 y[4] = {};
#pragma unroll
    for (int term = 0; term < 2; ++term) {
      bf16x8 bo[8];
#pragma unroll
      for (int r = 0; r < 64; ++r) {
        const bf16_t part = static_cast<bf16_t>(o[r >> 4][r & 15]);
        bo[r >> 3][r & 7] = part;
        o[r >> 4][r & 15] -= static_cast<float>(part);
      }
      hadamard_pairs(bo, y, lane);
    }
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      const u32x2 sg = *reinterpret_cast<const u32x2*>(a.signs_v + h * kGroup + 16 * s + 8 * hf);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        o[s >> 1][8 * (s & 1) + i] = __uint_as_float(__float_as_uint(y[s >> 1][8 * (s & 1) + i]) ^ ((i < 4 ? sg.x : sg.y) << (24 - 8 * (i & 3)) & 0x80000000u));
    }
  }
  if (!row_there) return;
  bf16_t* const out = static_cast<bf16_t*>(a.out) + ((w.first + qi) * a.q_heads + qh) * kGroup + 8 * hf;
#pragma unroll
  for (int s = 0; s < 8; ++s) {
    u32x4 x;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = Storage<bf16_t>::pack2(o[s >> 1][8 * (s & 1) + 2 * i], o[s >> 1][8 * (s & 1) + 2 * i + 1]);
    *reinterpret_cast<u32x4*>(out + 16 * s) = x;
  }
}

template <bool TREE> hipError_t launch_tiles(int n_codewords, const PagedAttendArgs& a, hipStream_t stream) {
  const dim3 grid = TREE ? dim3((unsigned)(a.H * a.items), (unsigned)a.row_blocks) : dim3((unsigned)(a.H * a.slots * a.row_blocks), (unsigned)a.batch);
#define AQUAKV_TILES(NCW) paged_tiles_kernel<NCW, TREE><<<grid, 64 * kTileWaves, 0, stream>>>(a)
  switch (n_codewords) {
    case kRtn2: AQUAKV_TILES(kRtn2); break;
    case kRtn4: AQUAKV_TILES(kRtn4); break;
    case 16: AQUAKV_TILES(16); break;
    case 64: AQUAKV_TILES(64); break;
    default: AQUAKV_TILES(256);
  }
#undef AQUAKV_TILES
  return hipGetLastError();
}

}  // namespace paged
}  // namespace aquakv
