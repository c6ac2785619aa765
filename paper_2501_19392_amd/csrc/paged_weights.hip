// The attention weight that each cached token gets: mass_t = keep mass_t + sum of softmax(scale q K^T)_t over the queries and the query heads of a kv head, from the
// codes of the keys as they are (paged_attend.h).  Operands are held as two fp16 numbers whatever the layer's type (22 bits, three products), as the
// sums come out in 32 bits.
#include "paged_rows.h"

#include <algorithm>

namespace aquakv {
namespace {

using namespace paged;

constexpr int kFewRows = kWeightsFewRows;                  // of a kv head, whose scores are kept (else they are taken again)
constexpr int kMassWaves = 4, kStaged = 2, kBehind = 4 * kStaged, kMassTokens = kTile * kMassWaves;      // of a workgroup that takes many rows

struct WeightsArgs {
  float* scores;                                           // few rows: [batch, H, rows, room], powers of two
  f32x2* stats;                                            // few rows: [items, H, rows], many: [batch, H, row tiles, token tiles, 16]: reference, sum
  int2* heads;                                             // few rows: [batch]: first item, items
  struct Row { float f, qsum0, qsum1, none; float ref, inv, pad[2]; };
  struct Packed { u32x4 q[2][4][64]; Row rows[16]; };      // operands of 16 rows [term][piece][lane], and the rows' numbers
  Packed* packed;                                          // many rows: [batch, H, row tiles]
  float* mass;
  float keep;
  int row_cap, tiles, room;                                // max_queries * (q_heads / H); row tiles; table_pages * page_tokens
};

// A row's query as operands: rotated, a power of two that brings it to fp16's range taken off.  f: what a product times the token's scale is to be multiplied by.
template <typename T, int NCW> __device__ __forceinline__ void query_operands(const PagedAttendArgs& a, const typename Codes<NCW, 2>::template Query<T>& asked, int c_exp,
                                                                              int lane, f16x8 (&q)[2][4], float (&qsum)[2], float& f) {
  typedef Codes<NCW, 2> C;
  constexpr bool kRtn = is_rtn(NCW);
  float v[32];
  C::template rotate_query<T>(asked, lane, v);
  const float by = a.scale * 1.4426950408889634f * (kRtn ? 1.0f : kRsqrtG);
  float top = 0.f;
#pragma unroll
  for (int r = 0; r < 32; ++r) top = fmaxf(top, fabsf(v[r]));
  const int e = max(__builtin_amdgcn_frexp_expf(column_max(top) * fabsf(by)), -100);
  f = __builtin_ldexpf(1.0f, min(e - kQueryExp + (kRtn ? C::kFieldExp : c_exp), 126));
  const float scaled = __builtin_ldexpf(by, kQueryExp - e);
#pragma unroll
  for (int r = 0; r < 32; ++r) v[r] *= scaled;
  C::pack_query(v, q, qsum);
}

// Uniform codes of piece j of the coordinates as an operand (as in Codes::scores).
template <typename C> __device__ __forceinline__ f16x8 code_operand(const uint32_t (&x)[4], int j) {
  const uint32_t d = C::kFields == 2 ? x[j] : (j & 1) ? x[j >> 1] >> 8 : x[j >> 1];
  uint32_t y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = C::kFields == 2 ? C::field((i & 2) ? d >> 8 : d, i & 1) : C::field(d, i);
  return operand(y[0], y[1], y[2], y[3]);
}

// Bound by memory and the vector pipes alike: 32 x 16 384 tokens, 4 heads a kv head, 63 us for 200 MB of codes and 48 MB of scores, 3.9 TB/s; with the codes in the caches it takes
// 50.  (Both terms of the query in operands of their own, 32 or 24 products a tile: 75 us.)  Scores are kept as they are a quarter of the codes: taking them again would read
// those a second time.
// Few rows: scores and statistics, one wave a piece of one kv head, as in paged_rows.h, but that a row has two columns: m its query's first terms, m + 8 the second
// ones.  A product with a key's operands then gives what both are to be added up from, and the two lanes share the eight tokens of their columns: 16 products a tile for 32.
// A look-up in a grid reads both terms of a point with one instruction (8 bytes a lane, all banks) and leaves them side by side in the operand, {point 0, its rest, point 1,
// its rest}: the query's pairs of coordinates are there twice instead.
template <int NCW> struct ScoreShape {
  static constexpr int kWaves = is_rtn(NCW) ? 4 : 8, kPerSimd = 4;
  static constexpr int kThreads = 64 * kWaves, kSlots = 256 * 4 * kPerSimd;
};
template <typename T, int NCW, bool FAR>
__global__ __launch_bounds__((ScoreShape<NCW>::kThreads)) __attribute__((amdgpu_waves_per_eu((ScoreShape<NCW>::kPerSimd)))) void
weights_scores_kernel(const PagedAttendArgs a, const WeightsArgs x) {
  constexpr int kWaves = ScoreShape<NCW>::kWaves;
  constexpr bool kRtn = is_rtn(NCW);
  typedef Codes<NCW, 2> C;
  __shared__ __align__(256) unsigned char lds[(kRtn ? 16 : C::kTableBytes) + kWaves * C::kScaleBytes];
  const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  unsigned char* const scale_lds = lds + (kRtn ? 16 : C::kTableBytes) + wave * C::kScaleBytes;
  const typename C::Points points = C::request_points(a.codebook, lane);
  const unsigned unit = blockIdx.x * kWaves + wave;
  const int h = uniform(unit % a.H), item = uniform(unit / a.H);
  const Share share = share_of(a, lane, item);
  if ((int)(blockIdx.x * kWaves / a.H) >= share.items) return;
  const int b = max(share.b, 0), rep = a.q_heads / a.H;
  const PagedQueries w = paged_queries(a, b);
  const int n_rows = w.n * rep, past = w.len - w.count;
  const bool idle = share.b < 0 || n_rows == 0;
  const int first_limit = past, last_limit = uniform(past + (n_rows - 1) / rep);
  const TokenRange range = piece_range(share.piece, share.tiles, kTile, idle ? 0 : last_limit + 1);
  const int t_begin = range.begin, t_end = range.end;
  int limit = -1;
  typename C::template Query<T> asked = {};
  if (!idle) {                                             // (rows that are not there: the last one again)
    const int there = min(m & 7, n_rows - 1), qi = there / rep, qh = h * rep + there % rep;
    limit = past + qi;
    asked = C::template request_query<T>(static_cast<const T*>(a.q) + (w.first + qi) * a.q_stride + qh * kGroup, a.signs_k, h, g);
  }
  // Keys are requested two tiles ahead, the rows that they are in three ahead.
  struct Tile { typename C::Keys k; unsigned there; };
  Tile s0 = {}, s1 = {}, s2 = {};
  Rows ahead = {};
  const auto request = [&](Tile& tile, const Rows& r, int t) {
    tile.there = there_of(r);
    if (t < t_end) tile.k = C::template request_keys<FAR, false>(a, r, h, lane);
  };
  if (t_begin < t_end) {
    request(s0, rows_of(a, b, t_begin), t_begin);
    request(s1, rows_of(a, b, t_begin + kTile), t_begin + kTile);
    ahead = rows_of(a, b, t_begin + 2 * kTile);
  }
  const int c_exp = C::template stage<kWaves>(points, lds, lane, wave);
  __syncthreads();
  if (idle) return;
  constexpr int kParts = kRtn ? 1 : 2;                     // operands that a piece of the coordinates takes
  f16x8 q[4][kParts];
  float qsum[2], f;
  {
    f16x8 both[2][4];
    query_operands<T, NCW>(a, asked, c_exp, lane, both, qsum, f);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const u32x4 hi = __builtin_bit_cast(u32x4, both[0][j]), lo = __builtin_bit_cast(u32x4, both[1][j]);
      u32x4 y;
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = m < 8 ? hi[i] : lo[i];
      if constexpr (kRtn) {
        q[j][0] = __builtin_bit_cast(f16x8, y);
      } else {
        q[j][0] = operand(y.x, y.x, y.y, y.y);
        q[j][1] = operand(y.z, y.z, y.w, y.w);
      }
    }
  }
  float ref = -3.0e38f, sum = 0.f;
  const int first = 8 * g + 4 * (m >> 3);                  // the lane's four tokens of a tile
  float* const to = x.scores + (((int64_t)b * a.H + h) * x.row_cap + (m & 7)) * x.room + first;
  const auto step = [&](const Tile& tile, int t, Tile& next) {
    if (t >= t_end) return;
    request(next, ahead, t + 2 * kTile);
    ahead = rows_of(a, b, t + 3 * kTile);
    asm volatile("" ::: "memory");                         // (a wave's LDS accesses stay in order)
    C::put_scales(tile.k, scale_lds, lane);
    asm volatile("" ::: "memory");
    f32x4 s[C::kHalves][2] = {};
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const uint32_t w4[4] = {tile.k.k[p].x, tile.k.k[p].y, tile.k.k[p].z, tile.k.k[p].w};
        if constexpr (kRtn) {
          s[j >> 1][p] = mfma(code_operand<C>(w4, j), q[j][0], s[j >> 1][p]);
        } else {
          u32x2 y[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) y[i] = *reinterpret_cast<const u32x2*>(lds + C::offset(w4, 4 * j + i, C::lane_copy(lane)));
          s[0][p] = mfma(operand(y[0].x, y[0].y, y[1].x, y[1].y), q[j][0], s[0][p]);
          s[0][p] = mfma(operand(y[2].x, y[2].y, y[3].x, y[3].y), q[j][kParts - 1], s[0][p]);
        }
      }
    // product p has the tokens 8 g + 4 p ...: the lane's own p is m / 8, the other one's goes to the lane of the row's other column
    float y[4];
    const auto four = [&](int row) { return *reinterpret_cast<const u32x2*>(scale_lds + 64 * row + 2 * first); };
    const auto half_of = [](const u32x2& w, int e) { return (float)__builtin_bit_cast(f16x2, e < 2 ? w.x : w.y)[e & 1]; };
    const auto int_of = [](const u32x2& w, int e) { return (float)(((e < 2 ? w.x : w.y) >> (16 * (e & 1))) & 0xffffu); };
#pragma unroll
    for (int k = 0; k < C::kHalves; ++k) {
      const u32x2 step = four(C::kKeys + 2 * k);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float own = m < 8 ? s[k][0][e] : s[k][1][e], other = m < 8 ? s[k][1][e] : s[k][0][e];
        float z = own + row_xor8(other);
        if constexpr (kRtn) z = __fmaf_rn(-int_of(four(C::kKeys + 2 * k + 1), e), qsum[k], z);
        y[e] = k == 0 ? z * half_of(step, e) : __fmaf_rn(z, half_of(step, e), y[e]);
      }
    }
    if (t + kTile - 1 > first_limit || tile.there != 15u) {
      asm volatile("");
      const int seen = min(limit + 1 - (t + first), (tile.there >> g) & 1 ? w.len - (t + first) : 0);
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = e < seen ? y[e] : -INFINITY;
    }
    const float top = fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3]));
    if (__builtin_amdgcn_ballot_w64(__fmaf_rn(top, f, -ref) > kTopExp) != 0) {
      const float most = column_max(top * f), moved = fmaxf(ref, fmaxf(most, row_xor8(most)) - kStartExp);
      sum *= __builtin_amdgcn_exp2f(ref - moved);
      ref = moved;
    }
    float p[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      y[e] *= f;                                           // (a power of two: exact)
      p[e] = __builtin_amdgcn_exp2f(y[e] - ref);
    }
    sum += sum_of(p);
    if ((m & 7) < n_rows && t + first < x.room) *reinterpret_cast<f32x4*>(to + t) = f32x4{y[0], y[1], y[2], y[3]};
  };
#pragma unroll 1
  for (int t = t_begin; t < t_end; t += 3 * kTile) {
    step(s0, t, s2);
    step(s1, t + kTile, s0);
    step(s2, t + 2 * kTile, s1);
  }
  if (share.piece == 0 && h == 0 && lane == 0) x.heads[b] = int2{item, share.pieces};
  sum = column_sum(sum);
  sum += row_xor8(sum);
  if (g == 0 && m < n_rows) x.stats[((int64_t)item * a.H + h) * x.row_cap + m] = f32x2{ref, sum};
}

// Reference and 1 / sum (0: the row sees nothing) of one row from its pieces, by `lanes` neighbouring lanes: every one gets it.
template <int LANES> __device__ __forceinline__ f32x2 joined_stats(const f32x2* at, int64_t step, int pieces, int l) {
  float ref = -3.0e38f, sum = 0.f;
  for (int i = l; i < pieces; i += LANES) {
    const f32x2 s = at[i * step];
    const float top = fmaxf(ref, s.x);
    sum = __fmaf_rn(sum, __builtin_amdgcn_exp2f(ref - top), s.y * __builtin_amdgcn_exp2f(s.x - top));
    ref = top;
  }
#pragma unroll
  for (int d = 1; d < LANES; d <<= 1) {                    // (both lanes of a pair add the same two numbers in the same order: lower lane's first)
    const float r2 = __shfl_xor(ref, d), s2 = __shfl_xor(sum, d), top = fmaxf(ref, r2);
    const float mine = sum * __builtin_amdgcn_exp2f(ref - top), other = s2 * __builtin_amdgcn_exp2f(r2 - top);
    sum = mine + other;
    ref = top;
  }
  return f32x2{ref, sum == 0.f ? 0.f : 1.0f / sum};
}

// The place of 8 tokens of a sequence in the mass of a head, -1: their page is not in the pool.
__device__ __forceinline__ int64_t mass_place(const PagedAttendArgs& a, int b, int h, uint32_t group) {
  uint32_t page = (uint32_t)(((uint64_t)group * a.page_magic) >> 32), in = group - page * a.page_groups;
  if (in >= a.page_groups) { ++page; in -= a.page_groups; }
  const int at = page < (uint32_t)a.table_pages ? a.page_table[(int64_t)b * a.table_pages + page] : -1;
  return (uint32_t)at < (uint32_t)a.pool.n_pages ? ((int64_t)at * a.H + h) * a.pool.page_tokens + in * 8 : -1;
}

// Few rows: mass from the scores, 15.8 us for 72 MB (32 x 16 384 tokens), 4.6 TB/s; with scores requested when the statistics are joined 17.5.  blockIdx = (1024 tokens and kv head, sequence), four tokens a thread.
constexpr int kChunk = 1024, kFirstRows = 4;
__global__ __launch_bounds__(256) void weights_from_scores_kernel(const PagedAttendArgs a, const WeightsArgs x) {
  __shared__ f32x2 stat[kFewRows];
  const int b = blockIdx.y, h = blockIdx.x % a.H, chunk = blockIdx.x / a.H;
  const PagedQueries w = paged_queries(a, b);
  if (chunk * kChunk >= w.len || w.n == 0) return;
  const int rep = a.q_heads / a.H, n_rows = w.n * rep, past = w.len - w.count;
  const int t = chunk * kChunk + 4 * threadIdx.x;
  const float* from = x.scores + ((int64_t)b * a.H + h) * x.row_cap * x.room + t;
  f32x4 s[kFirstRows] = {}, old = {0.f, 0.f, 0.f, 0.f};    // requested before the statistics are joined
  int64_t place = -1;
  if (t < w.len) {
#pragma unroll
    for (int r = 0; r < kFirstRows; ++r) s[r] = *reinterpret_cast<const f32x4*>(from + (int64_t)min(r, n_rows - 1) * x.room);
    place = mass_place(a, b, h, (uint32_t)t / 8);
  }
  float* const to = x.mass + place + (t & 4);
  if (place >= 0 && x.keep != 0.f && t < past) old = *reinterpret_cast<const f32x4*>(to);
  {
    const int row = threadIdx.x >> 5;
    const int2 head = x.heads[b];
    const f32x2 joined = joined_stats<32>(x.stats + ((int64_t)head.x * a.H + h) * x.row_cap + min(row, n_rows - 1), (int64_t)a.H * x.row_cap, head.y, threadIdx.x & 31);
    if ((threadIdx.x & 31) == 0) stat[row] = joined;
  }
  __syncthreads();
  if (place < 0) return;
  f32x4 gained = {0.f, 0.f, 0.f, 0.f};
  const auto add = [&](const f32x4& s, int r) {
    const int seen = past + r / rep + 1 - t;               // so many of the four
    const f32x2 st = stat[r];
#pragma unroll
    for (int e = 0; e < 4; ++e) gained[e] = e < seen ? __fmaf_rn(__builtin_amdgcn_exp2f(s[e] - st.x), st.y, gained[e]) : gained[e];
  };
#pragma unroll
  for (int r = 0; r < kFirstRows; ++r)
    if (r < n_rows) add(s[r], r);
  for (int r = kFirstRows; r < n_rows; ++r) add(*reinterpret_cast<const f32x4*>(from + (int64_t)r * x.room), r);
  if (x.keep != 0.f && t < past) {
#pragma unroll
    for (int e = 0; e < 4; ++e) gained[e] = t + e < past ? __fmaf_rn(x.keep, old[e], gained[e]) : gained[e];
  }
  if (t + 4 <= w.len) {
    *reinterpret_cast<f32x4*>(to) = gained;
  } else {
    for (int e = 0; e < 4; ++e)
      if (t + e < w.len) to[e] = gained[e];
  }
}

// Many rows: their queries as operands.  One wave for 16 rows of a kv head: blockIdx = (row tile and kv head, sequence).
template <typename T, int NCW>
__global__ __launch_bounds__(64) void weights_rows_kernel(const PagedAttendArgs a, const WeightsArgs x) {
  typedef Codes<NCW, 2> C;
  const int lane = threadIdx.x, m = lane & 15, g = lane >> 4, b = blockIdx.y, h = blockIdx.x % a.H, tile = blockIdx.x / a.H;
  const PagedQueries w = paged_queries(a, b);
  const int rep = a.q_heads / a.H, n_rows = w.n * rep, there = min(16 * tile + m, n_rows - 1), qi = there / rep, qh = h * rep + there % rep;
  if (16 * tile >= n_rows) return;
  const typename C::template Query<T> asked = C::template request_query<T>(static_cast<const T*>(a.q) + (w.first + qi) * a.q_stride + qh * kGroup, a.signs_k, h, g);
  int c_exp = 0;
  if constexpr (!is_rtn(NCW)) {                            // the grid's exponent, as stage() takes it
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < (2 * NCW + 63) / 64; ++i) top = fmaxf(top, fabsf(a.codebook[min(64 * i + lane, 2 * NCW - 1)]));
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
    c_exp = max(__builtin_amdgcn_frexp_expf(top), -100);
  }
  f16x8 q[2][4];
  float qsum[2], f;
  query_operands<T, NCW>(a, asked, c_exp, lane, q, qsum, f);
  const int64_t to = ((int64_t)b * a.H + h) * x.tiles + tile;
#pragma unroll
  for (int n = 0; n < 2; ++n)
#pragma unroll
    for (int j = 0; j < 4; ++j) x.packed[to].q[n][j][lane] = __builtin_bit_cast(u32x4, q[n][j]);
  if (g == 0) {
    WeightsArgs::Row r = {};
    r.f = f; r.qsum0 = qsum[0]; r.qsum1 = qsum[1];
    x.packed[to].rows[m] = r;
  }
}

// Row tiles that see something of the 32 tokens from t on: from this one.
__device__ __forceinline__ int first_tile(int t, int past, int rep) { return max(t - past, 0) * rep / 16; }
__device__ __forceinline__ int64_t token_tiles(const WeightsArgs& x) { return (x.room + kTile - 1) / kTile; }

// Many rows: a wave has 32 tokens of a kv head as operands, which take their conversion once, and goes through the row tiles, whose operands its workgroup brings to LDS,
// kStaged of them while the ones before are multiplied.  First for the statistics of the rows over its tokens, then, when those are joined, for the weights.
// 64 queries of 4 heads a kv head over 12 288 tokens: 25.4 and 23.9 us, of which 6 are the way in; matrix cores busy in 42 % of the cycles, vector pipes in 50, LDS in 35, of which
// 22 % are bank conflicts; a wave's products and exponentials follow each other.  (Row tiles requested behind a bound or a branch: 28 and 25; operands straight from the caches: 31 and 30.)
// The grid is there once (look-ups are few, and meet in banks as they will): a CU has three workgroups, by LDS (42 to 44 KB each) as by registers.  blockIdx = (128 tokens and kv head, sequence).
template <int NCW, bool MASS>
__global__ __launch_bounds__(64 * kMassWaves) __attribute__((amdgpu_waves_per_eu(3))) void weights_tokens_kernel(const PagedAttendArgs a, const WeightsArgs x) {
  typedef Codes<NCW, 2> C;
  constexpr bool kRtn = is_rtn(NCW);
  constexpr int kTable = kRtn ? 16 : NCW * 8, kTerms = kRtn ? 1 : 2, kThreads = 64 * kMassWaves;
  constexpr int kUnits = sizeof(WeightsArgs::Packed) / 16 * kStaged, kEach = (kUnits + kThreads - 1) / kThreads;
  __shared__ __align__(256) unsigned char table[kTable];
  __shared__ __align__(256) unsigned char scale_space[kMassWaves * C::kScaleBytes];
  __shared__ union { WeightsArgs::Packed tiles[kStaged]; u32x4 units[kEach * kThreads]; } staged[2];
  const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  unsigned char* const scale_lds = scale_space + wave * C::kScaleBytes;
  const int b = blockIdx.y, h = blockIdx.x % a.H, t0 = (blockIdx.x / a.H) * kMassTokens, t = t0 + wave * kTile;
  const PagedQueries w = paged_queries(a, b);
  if (t0 >= w.len || w.n == 0) return;
  const int rep = a.q_heads / a.H, n_rows = w.n * rep, past = w.len - w.count, tiles = (n_rows + 15) / 16;
  const int first = min(first_tile(t0, past, rep), tiles); // (later tokens' first row tiles are no earlier; the sequence may have more rows than are answered)
  const int64_t head = ((int64_t)b * a.H + h) * x.tiles;
  struct Coming { u32x4 x[kEach]; };
  Coming even, odd;
  // (Neither has a branch or a bound: loads wait for each other across the one, and the other is work, more than the 192 units of a stage's 1280 that are brought beside
  // its row tiles'.  There is room for kBehind row tiles behind the last one.)
  const auto request = [&](Coming& coming, int tile) {
    const u32x4* const at = reinterpret_cast<const u32x4*>(x.packed + head + tile);
#pragma unroll
    for (int i = 0; i < kEach; ++i) coming.x[i] = at[(unsigned)(i * kThreads) + threadIdx.x];
  };
  const auto put = [&](const Coming& coming, int buffer) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) staged[buffer].units[i * kThreads + threadIdx.x] = coming.x[i];
  };
  request(even, first);
  request(odd, first + kStaged);
  const typename C::Points points = C::request_points(a.codebook, lane);
  const Rows r = rows_of(a, b, t);                         // (a wave behind the sequence: its pages, if any, are read and not used)
  const typename C::Keys keys = C::template request_keys<true, false>(a, r, h, lane);
  if constexpr (!kRtn) {
    const int e = C::exponent(points);
    if (wave == 0) {
#pragma unroll
      for (int i = 0; i < C::kPoints; ++i) {
        if (lane >= NCW / C::kPoints) break;
        const float px = __builtin_ldexpf(points.x[2 * i], -e), py = __builtin_ldexpf(points.x[2 * i + 1], -e);
        uint32_t hi = f16_pair(px, py);
        asm("" : "+v"(hi));                                // (as in split_f16)
        const f16x2 top = __builtin_bit_cast(f16x2, hi);
        *reinterpret_cast<u32x2*>(table + 8 * (C::kPoints * lane + i)) = u32x2{hi, f16_pair(px - (float)top[0], py - (float)top[1])};
      }
    }
  }
  C::put_scales(keys, scale_lds, lane);
  put(even, 0);
  __syncthreads();
  f16x8 k[2][4][kTerms];                                   // [product][piece of the coordinates][term]
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const uint32_t y[4] = {keys.k[p].x, keys.k[p].y, keys.k[p].z, keys.k[p].w};
    if constexpr (kRtn) {
#pragma unroll
      for (int j = 0; j < 4; ++j) k[p][j][0] = code_operand<C>(y, j);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        u32x2 o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = *reinterpret_cast<const u32x2*>(table + (C::offset(y, 4 * j + i, 0u) >> 5));
        k[p][j][0] = operand(o[0].x, o[1].x, o[2].x, o[3].x);
        k[p][j][kTerms - 1] = operand(o[0].y, o[1].y, o[2].y, o[3].y);
      }
    }
  }
  const unsigned there = there_of(r);
  const int held = (there >> g) & 1 ? w.len - (t + 8 * g) : 0;
  float gained[8] = {};
  f32x2* const stats = x.stats + (head * token_tiles(x) + t / kTile) * 16 + m;
  float sigma[8];                                          // grids: the scales of the lane's tokens
  if constexpr (!kRtn) {
    const u32x4 ks = C::eight(scale_lds, C::kKeys, g);
#pragma unroll
    for (int e = 0; e < 8; ++e) sigma[e] = C::half_at(ks, e);
  }
  const auto finish = [&](const f32x4 (&s)[C::kHalves][2], const WeightsArgs::Row& row, int tile) {
    const float f = row.f, qsum[2] = {row.qsum0, row.qsum1};
    float y[8];
    if constexpr (kRtn) {
      C::scaled(s, scale_lds, g, qsum, y);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = s[0][e >> 2][e & 3] * sigma[e];
    }
    if (t + kTile - 1 > past + 16 * tile / rep || there != 15u) {
      asm volatile("");
      const int mine = 16 * tile + m, seen = mine < n_rows ? min(past + mine / rep + 1 - (t + 8 * g), held) : 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = e < seen ? y[e] : -INFINITY;
      if constexpr (MASS) {                                // (a row without numbers reaches no token that it does not see)
        const float ref = row.ref, inv = row.inv;
#pragma unroll
        for (int e = 0; e < 8; ++e) gained[e] = e < seen ? __fmaf_rn(__builtin_amdgcn_exp2f(__fmaf_rn(y[e], f, -ref)), inv, gained[e]) : gained[e];
        return;
      }
    }
    if constexpr (MASS) {
      const float ref = row.ref, inv = row.inv;
#pragma unroll
      for (int e = 0; e < 8; ++e) gained[e] = __fmaf_rn(__builtin_amdgcn_exp2f(__fmaf_rn(y[e], f, -ref)), inv, gained[e]);
    } else {
      float top = y[0];
#pragma unroll
      for (int e = 1; e < 8; ++e) top = fmaxf(top, y[e]);
      const float most = fmaxf(column_max(top) * f, -3.0e38f);
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = __builtin_amdgcn_exp2f(__fmaf_rn(y[e], f, -most));
      const float sum = column_sum(sum_of(p));
      if (g == 0) stats[(int64_t)tile * token_tiles(x) * 16] = f32x2{most, sum};
    }
  };
  const int from = first_tile(t, past, rep);
  // A stage is requested two stages ahead: what another chiplet wrote takes longer than one.
  const auto stage_of = [&](int tile, int buffer, Coming& next, const Coming& behind) {
    request(next, tile + 2 * kStaged);
    if (t < w.len) {
      // products of kStaged row tiles and two halves of the tokens in turn (a product waits for the last one of its own); of a row tile that is not there, anything
      f32x4 s[kStaged][C::kHalves][2] = {};
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          f16x8 q[kStaged];
#pragma unroll
          for (int i = 0; i < kStaged; ++i) q[i] = __builtin_bit_cast(f16x8, staged[buffer].tiles[i].q[n][j][lane]);
#pragma unroll
          for (int term = 0; term < (n == 0 ? kTerms : 1); ++term)
#pragma unroll
            for (int i = 0; i < kStaged; ++i)
#pragma unroll
              for (int p = 0; p < 2; ++p) {
                f32x4& y = s[i][kRtn ? j >> 1 : 0][p];
                y = mfma(k[p][j][term], q[i], y);
              }
        }
      // operands are read two steps ahead of their products
      constexpr int kFirst = 2 * kTerms * kStaged, kSecond = 2 * kStaged;
#define AQUAKV_STEP(MFMAS, READS) __builtin_amdgcn_sched_group_barrier(0x008, MFMAS, 0); __builtin_amdgcn_sched_group_barrier(0x100, READS, 0)
      __builtin_amdgcn_sched_group_barrier(0x100, 2 * kStaged, 0);
      AQUAKV_STEP(kFirst, kStaged); AQUAKV_STEP(kSecond, kStaged); AQUAKV_STEP(kFirst, kStaged);
      AQUAKV_STEP(kSecond, kStaged); AQUAKV_STEP(kFirst, kStaged); AQUAKV_STEP(kSecond, kStaged);
#undef AQUAKV_STEP
      __builtin_amdgcn_sched_group_barrier(0x008, kFirst + kSecond, 0);
#pragma unroll
      for (int i = 0; i < kStaged; ++i)
        if (tile + i >= from && tile + i < tiles) finish(s[i], staged[buffer].tiles[i].rows[m], tile + i);
    }
    put(behind, buffer ^ 1);
    __syncthreads();
  };
#pragma unroll 1
  for (int tile = first; tile < tiles; tile += 2 * kStaged) {
    stage_of(tile, 0, even, odd);
    if (tile + kStaged >= tiles) break;
    stage_of(tile + kStaged, 1, odd, even);
  }
  if (t >= w.len) return;
  if constexpr (MASS) {
    // sums over the 16 rows of a lane group; lane m < 8 has token 8 g + m
    float mine = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float y = gained[e];
      y += quad_xor<1>(y);
      y += quad_xor<2>(y);
      y += octet_mirror(y);
      y += row_xor8(y);
      mine = m == e ? y : mine;
    }
    const int token = t + 8 * g + m;
    if (m >= 8 || m >= held) return;
    const int64_t place = mass_place(a, b, h, (uint32_t)(t / 8 + g));
    float* const to = x.mass + place + m;
    if (x.keep != 0.f && token < past) mine = __fmaf_rn(x.keep, *to, mine);
    *to = mine;
  }
}

// Many rows: the statistics of a row tile over all token tiles.  blockIdx = (row tile and kv head, sequence); wave w takes token tiles 4 w + g, 4 w + g + 16, ...
__global__ __launch_bounds__(256) void weights_join_kernel(const PagedAttendArgs a, const WeightsArgs x) {
  __shared__ f32x2 part[4][16];
  const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4, wave = threadIdx.x >> 6, b = blockIdx.y, h = blockIdx.x % a.H, tile = blockIdx.x / a.H;
  const PagedQueries w = paged_queries(a, b);
  const int rep = a.q_heads / a.H, n_rows = w.n * rep, past = w.len - w.count, n = tiles_of_tokens(w.len, kTile);
  if (16 * tile >= n_rows) return;
  const int64_t at = ((int64_t)b * a.H + h) * x.tiles + tile;
  const f32x2* const from = x.stats + at * token_tiles(x) * 16 + m;
  float ref = -3.0e38f, sum = 0.f;
#pragma unroll 8
  for (int i = 4 * wave + g; i < n; i += 16) {             // (tiles that this row tile was left out of are the last ones)
    f32x2 s = {-3.0e38f, 0.f};
    if (tile >= first_tile(i * kTile, past, rep)) s = from[(int64_t)i * 16];
    const float top = fmaxf(ref, s.x);
    sum = __fmaf_rn(sum, __builtin_amdgcn_exp2f(ref - top), s.y * __builtin_amdgcn_exp2f(s.x - top));
    ref = top;
  }
  const float all = column_max(ref);
  sum = column_sum(sum * __builtin_amdgcn_exp2f(ref - all));
  if (g == 0) part[wave][m] = f32x2{all, sum};
  __syncthreads();
  if (threadIdx.x >= 16) return;
  float top = part[0][m].x, total = 0.f;
#pragma unroll
  for (int i = 1; i < 4; ++i) top = fmaxf(top, part[i][m].x);
#pragma unroll
  for (int i = 0; i < 4; ++i) total = __fmaf_rn(part[i][m].y, __builtin_amdgcn_exp2f(part[i][m].x - top), total);
  WeightsArgs::Row& row = x.packed[at].rows[m];
  row.ref = top;
  row.inv = total == 0.f || 16 * tile + m >= n_rows ? 0.f : 1.0f / total;      // (rows that are not there: the last one again, which adds nothing)
}

struct WeightsPlan { bool few; unsigned blocks; int slots, rows; int64_t room; size_t scores, stats, heads, packed; };
template <int NCW> WeightsPlan weights_plan(const PagedAttendArgs& a) {
  WeightsPlan p = {};
  const int64_t rows = std::max<int64_t>(a.max_queries, 1) * (a.q_heads / a.H), room = (int64_t)a.table_pages * a.pool.page_tokens, most = (room + kTile - 1) / kTile;
  const auto padded = [](int64_t n) { return ((size_t)n + 255) & ~(size_t)255; };
  const int64_t heads = (int64_t)a.batch * a.H, tiles = (rows + 15) / 16;
  p.few = rows <= kFewRows;
  p.rows = (int)rows;
  p.room = room;
  if (p.few) {
    p.slots = std::max(ScoreShape<NCW>::kSlots / a.H, 1);
    const int64_t items = std::min(a.batch * std::max<int64_t>(most, 1), std::max<int64_t>(p.slots - a.batch, std::max(p.slots / 2, 1)) + a.batch);
    p.blocks = (unsigned)((items * a.H + ScoreShape<NCW>::kWaves - 1) / ScoreShape<NCW>::kWaves);
    p.scores = padded(heads * rows * room * sizeof(float));
    p.stats = padded(items * a.H * rows * sizeof(f32x2));
    p.heads = padded(a.batch * (int64_t)sizeof(int2));
  } else {
    p.stats = padded(heads * tiles * most * 16 * sizeof(f32x2));
    p.packed = padded((heads * tiles + kBehind) * sizeof(WeightsArgs::Packed));
  }
  return p;
}
WeightsPlan plan_of(int n_codewords, const PagedAttendArgs& a) {
  WeightsPlan p = {};
  AQUAKV_PAGED_N(n_codewords, (p = weights_plan<N>(a)));
  return p;
}

}  // namespace

size_t paged_weights_workspace_bytes(int n_codewords, const PagedAttendArgs& a) {
  const WeightsPlan p = plan_of(n_codewords, a);
  return p.scores + p.stats + p.heads + p.packed;
}

hipError_t launch_paged_weights(int dtype, int n_codewords, const PagedAttendArgs& args, float keep, float* mass, void* workspace, hipStream_t stream) {
  PagedAttendArgs a = args;
  const WeightsPlan plan = plan_of(n_codewords, a);
  a.slots = plan.slots;
  a.page_groups = a.pool.page_tokens / 8;
  a.page_magic = a.page_groups == 1 ? 0xffffffffu : (uint32_t)((uint64_t(1) << 32) / a.page_groups);
  WeightsArgs x = {};
  unsigned char* at = static_cast<unsigned char*>(workspace);
  const auto take = [&](size_t n) { unsigned char* const p = at; at += n; return p; };
  x.scores = reinterpret_cast<float*>(take(plan.scores));
  x.stats = reinterpret_cast<f32x2*>(take(plan.stats));
  x.heads = reinterpret_cast<int2*>(take(plan.heads));
  x.packed = reinterpret_cast<WeightsArgs::Packed*>(take(plan.packed));
  x.mass = mass; x.keep = keep;
  x.row_cap = plan.rows; x.tiles = (plan.rows + 15) / 16; x.room = (int)plan.room;
  if (plan.few) {
    const bool far = (uint64_t)a.pool.rows * a.H * (kGroup / 2) > 0xffffffffull;
    AQUAKV_PAGED(dtype, n_codewords, (far ? weights_scores_kernel<T, N, true><<<plan.blocks, ScoreShape<N>::kThreads, 0, stream>>>(a, x)
                                          : weights_scores_kernel<T, N, false><<<plan.blocks, ScoreShape<N>::kThreads, 0, stream>>>(a, x)));
    if (const hipError_t e = hipGetLastError()) return e;
    weights_from_scores_kernel<<<dim3((unsigned)((plan.room + kChunk - 1) / kChunk * a.H), (unsigned)a.batch), 256, 0, stream>>>(a, x);
    return hipGetLastError();
  }
  const dim3 tiles((unsigned)(x.tiles * a.H), (unsigned)a.batch), tokens((unsigned)((plan.room + kMassTokens - 1) / kMassTokens * a.H), (unsigned)a.batch);
  AQUAKV_PAGED(dtype, n_codewords, (weights_rows_kernel<T, N><<<tiles, 64, 0, stream>>>(a, x)));
  if (const hipError_t e = hipGetLastError()) return e;
  AQUAKV_PAGED_N(n_codewords, (weights_tokens_kernel<N, false><<<tokens, 64 * kMassWaves, 0, stream>>>(a, x)));
  if (const hipError_t e = hipGetLastError()) return e;
  weights_join_kernel<<<tiles, 256, 0, stream>>>(a, x);
  if (const hipError_t e = hipGetLastError()) return e;
  AQUAKV_PAGED_N(n_codewords, (weights_tokens_kernel<N, true><<<tokens, 64 * kMassWaves, 0, stream>>>(a, x)));
  return hipGetLastError();
}

}  // namespace aquakv
