// The attention weight that each cached token gets: mass_t = keep mass_t + sum of softmax(scale q K^T)_t over the queries and the query heads of a kv head, from the
// codes of the keys as they are (paged_attend.h).  Operands are held as two fp16 numbers whatever the layer's type (22 bits, three products), as the
// sums come out in 32 bits.
#include "paged_rows.h"

#include <algorithm>

namespace aquakv {
namespace {

using namespace paged;

constexpr int kFewRows = 8;                                // of a kv head, whose scores are kept (else they are taken again)
constexpr int kMassWaves = 4, kMassTokens = kTile * kMassWaves;      // of a workgroup that takes many rows

struct WeightsArgs {
  float* scores;                                           // few rows: [batch, H, rows, room], powers of two
  f32x2* stats;                                            // [items, H, rows]: reference, sum
  int2* heads;                                             // [batch]: first item, items
  u32x4* packed;                                           // many rows: [batch, H, row tiles, term, piece, lane] operands of 16 rows
  struct Row { float f, qsum0, qsum1, ref, inv, pad[3]; }* rows;      // [batch, H, row tiles, 16]
  float* mass;
  float keep;
  int row_cap, tiles, room;                                // max_queries * (q_heads / H); row tiles; table_pages * page_tokens
};

// Scores and statistics of COLS columns of 16 rows: one wave a piece of one kv head, as in paged_rows.h.
template <typename T, int NCW, int COLS> struct ScoreShape {
  static constexpr int kWaves = is_rtn(NCW) ? 4 : 8, kPerSimd = COLS == 2 ? 3 : 4;
  static constexpr int kThreads = 64 * kWaves, kSlots = 256 * 4 * kPerSimd;
};
template <typename T, int NCW, int COLS, bool FAR>
__global__ __launch_bounds__((ScoreShape<T, NCW, COLS>::kThreads)) __attribute__((amdgpu_waves_per_eu((ScoreShape<T, NCW, COLS>::kPerSimd)))) void
weights_scores_kernel(const PagedAttendArgs a, const WeightsArgs x) {
  constexpr int kWaves = ScoreShape<T, NCW, COLS>::kWaves, kRows = 16 * COLS;
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
  const int n_rows = w.n * rep, row0 = blockIdx.y * kRows, past = w.len - w.count;
  const bool idle = share.b < 0 || row0 >= n_rows;
  const int first_limit = uniform(past + row0 / rep), last_limit = uniform(past + min(row0 + kRows - 1, n_rows - 1) / rep);
  const TokenRange range = piece_range(share.piece, share.tiles, kTile, idle ? 0 : last_limit + 1);
  const int t_begin = range.begin, t_end = range.end;
  const bool any = t_begin < t_end;
  struct { f16x8 q[2][4]; float qsum[2], f, ref, sum; int limit; } col[COLS];
  typename C::template Query<T> asked[COLS] = {};
  if (!idle) {
#pragma unroll
    for (int i = 0; i < COLS; ++i) {
      const int row = row0 + 16 * i + m, there = min(row, n_rows - 1), qi = there / rep, qh = h * rep + there % rep;
      col[i].limit = row < n_rows ? past + qi : -1;
      asked[i] = C::template request_query<T>(static_cast<const T*>(a.q) + (w.first + qi) * a.q_stride + qh * kGroup, a.signs_k, h, g);
    }
  }
  Rows r0 = {}, r1 = {};
  typename C::Keys k = {}, next = {};
  if (any) {
    r0 = rows_of(a, b, t_begin);
    r1 = rows_of(a, b, t_begin + kTile);
    k = C::template request_keys<FAR, false>(a, r0, h, lane);
  }
  const int c_exp = C::template stage<kWaves>(points, lds, lane, wave);
  __syncthreads();
  if (idle) return;
#pragma unroll
  for (int i = 0; i < COLS; ++i) {
    float v[32];
    C::template rotate_query<T>(asked[i], lane, v);
    const float by = a.scale * 1.4426950408889634f * (kRtn ? 1.0f : kRsqrtG);
    float top = 0.f;
#pragma unroll
    for (int r = 0; r < 32; ++r) top = fmaxf(top, fabsf(v[r]));
    const int e = max(__builtin_amdgcn_frexp_expf(column_max(top) * fabsf(by)), -100);
    col[i].f = __builtin_ldexpf(1.0f, min(e - kQueryExp + (kRtn ? C::kFieldExp : c_exp), 126));
    const float scaled = __builtin_ldexpf(by, kQueryExp - e);
#pragma unroll
    for (int r = 0; r < 32; ++r) v[r] *= scaled;
    C::pack_query(v, col[i].q, col[i].qsum);
    col[i].ref = -3.0e38f;
    col[i].sum = 0.f;
  }
#pragma unroll 1
  for (int t = t_begin; t < t_end; t += kTile) {
    const bool more = t + kTile < t_end;
    if (more) next = C::template request_keys<FAR, false>(a, r1, h, lane);
    const unsigned there = there_of(r0);
    const Rows r2 = rows_of(a, b, t + 2 * kTile);
    asm volatile("" ::: "memory");                         // (a wave's LDS accesses stay in order)
    C::put_scales(k, scale_lds, lane);
    asm volatile("" ::: "memory");
    f32x4 s[COLS][C::kHalves][2] = {};
#pragma unroll
    for (int p = 0; p < 2; ++p) C::scores(k, p, lds, lane, col, s);
    const int held = (there >> g) & 1 ? w.len - (t + 8 * g) : 0;
    const bool masked = t + kTile - 1 > first_limit || t + kTile > t_end || there != 15u;
#pragma unroll
    for (int i = 0; i < COLS; ++i) {
      float y[8];
      C::scaled(s[i], scale_lds, g, col[i].qsum, y);
      if (masked) {
        asm volatile("");
        const int seen = min(col[i].limit + 1 - (t + 8 * g), held);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = e < seen ? y[e] : -INFINITY;
      }
      float top = y[0];
#pragma unroll
      for (int e = 1; e < 8; ++e) top = fmaxf(top, y[e]);
      if (__builtin_amdgcn_ballot_w64(__fmaf_rn(top, col[i].f, -col[i].ref) > kTopExp) != 0) {
        const float moved = fmaxf(col[i].ref, column_max(top * col[i].f) - kStartExp);
        col[i].sum *= __builtin_amdgcn_exp2f(col[i].ref - moved);
        col[i].ref = moved;
      }
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = __builtin_amdgcn_exp2f(__fmaf_rn(y[e], col[i].f, -col[i].ref));
      col[i].sum += sum_of(p);
      if constexpr (COLS == 1) {                           // (times a power of two: exact)
        const int at = t + 8 * g;
        if (m < n_rows && at < x.room) {
          float* const to = x.scores + (((int64_t)b * a.H + h) * x.row_cap + m) * x.room + at;
          *reinterpret_cast<f32x4*>(to) = f32x4{y[0], y[1], y[2], y[3]} * col[i].f;
          *reinterpret_cast<f32x4*>(to + 4) = f32x4{y[4], y[5], y[6], y[7]} * col[i].f;
        }
      }
    }
    k = next;
    r0 = r1;
    r1 = r2;
  }
  if (share.piece == 0 && h == 0 && blockIdx.y == 0 && lane == 0) x.heads[b] = int2{item, share.pieces};
#pragma unroll
  for (int i = 0; i < COLS; ++i) {
    const float sum = column_sum(col[i].sum);
    const int row = row0 + 16 * i + m;
    if (g == 0 && row < n_rows) x.stats[((int64_t)item * a.H + h) * x.row_cap + row] = f32x2{col[i].ref, sum};
  }
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

// Few rows: mass from the scores.  blockIdx = (1024 tokens and kv head, sequence), four tokens a thread.
constexpr int kChunk = 1024;
__global__ __launch_bounds__(256) void weights_from_scores_kernel(const PagedAttendArgs a, const WeightsArgs x) {
  __shared__ f32x2 stat[kFewRows];
  const int b = blockIdx.y, h = blockIdx.x % a.H, chunk = blockIdx.x / a.H;
  const PagedQueries w = paged_queries(a, b);
  if (chunk * kChunk >= w.len || w.n == 0) return;
  const int rep = a.q_heads / a.H, n_rows = w.n * rep, past = w.len - w.count;
  {
    const int row = threadIdx.x >> 5;
    const int2 head = x.heads[b];
    const f32x2 s = joined_stats<32>(x.stats + ((int64_t)head.x * a.H + h) * x.row_cap + min(row, n_rows - 1), (int64_t)a.H * x.row_cap, head.y, threadIdx.x & 31);
    if ((threadIdx.x & 31) == 0) stat[row] = s;
  }
  __syncthreads();
  const int t = chunk * kChunk + 4 * threadIdx.x;
  if (t >= w.len) return;
  const int64_t place = mass_place(a, b, h, (uint32_t)t / 8);
  if (place < 0) return;
  float* const to = x.mass + place + (t & 4);
  f32x4 gained = {0.f, 0.f, 0.f, 0.f};
  const float* from = x.scores + ((int64_t)b * a.H + h) * x.row_cap * x.room + t;
  for (int r = 0; r < n_rows; ++r, from += x.room) {
    const int seen = past + r / rep + 1 - t;               // so many of the four
    if (seen <= 0) continue;
    const f32x4 s = *reinterpret_cast<const f32x4*>(from);
    const f32x2 st = stat[r];
#pragma unroll
    for (int e = 0; e < 4; ++e) gained[e] = __fmaf_rn(e < seen ? __builtin_amdgcn_exp2f(s[e] - st.x) : 0.f, st.y, gained[e]);
  }
  if (x.keep != 0.f && t < past) {
    const f32x4 old = *reinterpret_cast<const f32x4*>(to);
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

// Many rows: their statistics joined, their queries as operands.  One wave for 16 rows of a kv head: blockIdx = (row tile and kv head, sequence).
template <typename T, int NCW>
__global__ __launch_bounds__(64) void weights_rows_kernel(const PagedAttendArgs a, const WeightsArgs x) {
  typedef Codes<NCW, 2> C;
  constexpr bool kRtn = is_rtn(NCW);
  const int lane = threadIdx.x, m = lane & 15, g = lane >> 4, b = blockIdx.y, h = blockIdx.x % a.H, tile = blockIdx.x / a.H;
  const PagedQueries w = paged_queries(a, b);
  const int rep = a.q_heads / a.H, n_rows = w.n * rep, row = 16 * tile + m, there = min(row, n_rows - 1), qi = there / rep, qh = h * rep + there % rep;
  if (16 * tile >= n_rows) return;
  const typename C::template Query<T> asked = C::template request_query<T>(static_cast<const T*>(a.q) + (w.first + qi) * a.q_stride + qh * kGroup, a.signs_k, h, g);
  int c_exp = 0;
  if constexpr (!kRtn) {                                   // the grid's exponent, as stage() takes it
    float top = 0.f;
    for (int i = lane; i < 2 * NCW; i += 64) top = fmaxf(top, fabsf(a.codebook[i]));
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
    c_exp = max(__builtin_amdgcn_frexp_expf(top), -100);
  }
  const int2 head = x.heads[b];
  // lanes of a row are 16 apart here
  const f32x2* const at = x.stats + ((int64_t)head.x * a.H + h) * x.row_cap + there;
  float ref = -3.0e38f, sum = 0.f;
  for (int i = g; i < head.y; i += 4) {
    const f32x2 s = at[(int64_t)i * a.H * x.row_cap];
    const float top = fmaxf(ref, s.x);
    sum = __fmaf_rn(sum, __builtin_amdgcn_exp2f(ref - top), s.y * __builtin_amdgcn_exp2f(s.x - top));
    ref = top;
  }
  const float all = column_max(ref);
  sum = column_sum(sum * __builtin_amdgcn_exp2f(ref - all));
  float v[32];
  C::template rotate_query<T>(asked, lane, v);
  const float by = a.scale * 1.4426950408889634f * (kRtn ? 1.0f : kRsqrtG);
  float top = 0.f;
#pragma unroll
  for (int r = 0; r < 32; ++r) top = fmaxf(top, fabsf(v[r]));
  const int e = max(__builtin_amdgcn_frexp_expf(column_max(top) * fabsf(by)), -100);
  const float scaled = __builtin_ldexpf(by, kQueryExp - e);
#pragma unroll
  for (int r = 0; r < 32; ++r) v[r] *= scaled;
  f16x8 q[2][4];
  float qsum[2];
  C::pack_query(v, q, qsum);
  const int64_t to = ((int64_t)b * a.H + h) * x.tiles + tile;
#pragma unroll
  for (int n = 0; n < 2; ++n)
#pragma unroll
    for (int j = 0; j < 4; ++j) x.packed[(to * 8 + 4 * n + j) * 64 + lane] = __builtin_bit_cast(u32x4, q[n][j]);
  if (g == 0) {
    WeightsArgs::Row r = {};
    r.f = __builtin_ldexpf(1.0f, min(e - kQueryExp + (kRtn ? C::kFieldExp : c_exp), 126));
    r.qsum0 = qsum[0]; r.qsum1 = qsum[1]; r.ref = all; r.inv = sum == 0.f || row >= n_rows ? 0.f : 1.0f / sum;      // (rows that are not there: the last one again, which adds nothing)
    x.rows[to * 16 + m] = r;
  }
}

// Many rows: a wave has 32 tokens of a kv head as operands and takes the row tiles in turn.  blockIdx = (128 tokens and kv head, sequence).
template <int NCW>
__global__ __launch_bounds__(64 * kMassWaves) __attribute__((amdgpu_waves_per_eu(2))) void weights_mass_kernel(const PagedAttendArgs a, const WeightsArgs x) {
  typedef Codes<NCW, 2> C;
  constexpr bool kRtn = is_rtn(NCW);
  constexpr int kTable = kRtn ? 16 : C::kTableBytes, kTerms = kRtn ? 1 : 2;
  __shared__ __align__(256) unsigned char lds[kTable + kMassWaves * C::kScaleBytes];
  const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  unsigned char* const scale_lds = lds + kTable + wave * C::kScaleBytes;
  const int b = blockIdx.y, h = blockIdx.x % a.H, t0 = (blockIdx.x / a.H) * kMassTokens, t = t0 + wave * kTile;
  const PagedQueries w = paged_queries(a, b);
  if (t0 >= w.len || w.n == 0) return;
  const typename C::Points points = C::request_points(a.codebook, lane);
  const Rows r = rows_of(a, b, t);
  const typename C::Keys keys = C::template request_keys<true, false>(a, r, h, lane);
  C::template stage<kMassWaves>(points, lds, lane, wave);
  __syncthreads();
  if (t >= w.len) return;
  C::put_scales(keys, scale_lds, lane);
  asm volatile("" ::: "memory");
  f16x8 k[2][4][kTerms];                                   // [product][piece of the coordinates][term]
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const uint32_t y[4] = {keys.k[p].x, keys.k[p].y, keys.k[p].z, keys.k[p].w};
    if constexpr (kRtn) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t z[4];
        const uint32_t d = NCW == kRtn4 ? y[j] : (j & 1) ? y[j >> 1] >> 8 : y[j >> 1];
#pragma unroll
        for (int i = 0; i < 4; ++i) z[i] = NCW == kRtn4 ? C::field((i & 2) ? d >> 8 : d, i & 1) : C::field(d, i);
        k[p][j][0] = operand(z[0], z[1], z[2], z[3]);
      }
    } else {
      const uint32_t at = C::lane_copy(lane);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = C::offset(y, 4 * j + i, at);
        k[p][j][0] = operand(C::point(lds, o[0]), C::point(lds, o[1]), C::point(lds, o[2]), C::point(lds, o[3]));
        k[p][j][kTerms - 1] = operand(C::template point<1>(lds, o[0]), C::template point<1>(lds, o[1]), C::template point<1>(lds, o[2]), C::template point<1>(lds, o[3]));
      }
    }
  }
  const int rep = a.q_heads / a.H, n_rows = w.n * rep, past = w.len - w.count;
  const unsigned there = there_of(r);
  const int held = (there >> g) & 1 ? w.len - (t + 8 * g) : 0;
  float gained[8] = {};
  const int from = max(t - past, 0) * rep / 16, tiles = (n_rows + 15) / 16;      // (rows ahead of it see none of these tokens)
  const int64_t head = ((int64_t)b * a.H + h) * x.tiles;
  const u32x4* const packed = x.packed + head * 8 * 64 + lane;
  const WeightsArgs::Row* const rows = x.rows + head * 16 + m;
#pragma unroll 1
  for (int tile = from; tile < tiles; ++tile) {
    f16x8 q[2][4];
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int j = 0; j < 4; ++j) q[n][j] = __builtin_bit_cast(f16x8, packed[((int64_t)tile * 8 + 4 * n + j) * 64]);
    const WeightsArgs::Row row = rows[(int64_t)tile * 16];
    f32x4 s[C::kHalves][2] = {};
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        f32x4& y = s[kRtn ? j >> 1 : 0][p];
        y = mfma(k[p][j][0], q[0][j], y);
        y = mfma(k[p][j][0], q[1][j], y);
        if constexpr (!kRtn) y = mfma(k[p][j][1], q[0][j], y);
      }
    float y[8];
    const float qsum[2] = {row.qsum0, row.qsum1};
    C::scaled(s, scale_lds, g, qsum, y);
    if (t + kTile - 1 > past + 16 * tile / rep || there != 15u) {
      asm volatile("");
      const int mine = 16 * tile + m, seen = mine < n_rows ? min(past + mine / rep + 1 - (t + 8 * g), held) : 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = e < seen ? y[e] : -INFINITY;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) gained[e] = __fmaf_rn(__builtin_amdgcn_exp2f(__fmaf_rn(y[e], row.f, -row.ref)), row.inv, gained[e]);
  }
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

struct WeightsPlan { bool few; unsigned blocks, row_tiles; int slots, rows; int64_t items, room; size_t scores, stats, heads, packed, row_bytes; };
template <typename T, int NCW> WeightsPlan weights_plan(const PagedAttendArgs& a) {
  WeightsPlan p = {};
  const int64_t rows = std::max<int64_t>(a.max_queries, 1) * (a.q_heads / a.H), room = (int64_t)a.table_pages * a.pool.page_tokens, most = (room + kTile - 1) / kTile;
  p.few = rows <= kFewRows;
  p.rows = (int)rows;
  p.room = room;
  p.row_tiles = p.few ? 1 : (unsigned)((rows + 31) / 32);
  p.slots = (int)std::max<int64_t>((p.few ? ScoreShape<T, NCW, 1>::kSlots : ScoreShape<T, NCW, 2>::kSlots) / (a.H * (int64_t)p.row_tiles), 1);
  p.items = std::min(a.batch * std::max<int64_t>(most, 1), std::max<int64_t>(p.slots - a.batch, std::max(p.slots / 2, 1)) + a.batch);
  constexpr int kWaves = ScoreShape<T, NCW, 1>::kWaves;
  p.blocks = (unsigned)((p.items * a.H + kWaves - 1) / kWaves);
  const auto padded = [](int64_t n) { return ((size_t)n + 255) & ~(size_t)255; };
  const int64_t heads = (int64_t)a.batch * a.H, tiles = (rows + 15) / 16;
  p.scores = p.few ? padded(heads * rows * room * sizeof(float)) : 0;
  p.stats = padded(p.items * a.H * rows * sizeof(f32x2));
  p.heads = padded(a.batch * (int64_t)sizeof(int2));
  p.packed = p.few ? 0 : padded(heads * tiles * 8 * 64 * sizeof(u32x4));
  p.row_bytes = p.few ? 0 : padded(heads * tiles * 16 * sizeof(WeightsArgs::Row));
  return p;
}
WeightsPlan plan_of(int dtype, int n_codewords, const PagedAttendArgs& a) {
  WeightsPlan p = {};
  AQUAKV_PAGED(dtype, n_codewords, (p = weights_plan<T, N>(a)));
  return p;
}

}  // namespace

size_t paged_weights_workspace_bytes(int dtype, int n_codewords, const PagedAttendArgs& a) {
  const WeightsPlan p = plan_of(dtype, n_codewords, a);
  return p.scores + p.stats + p.heads + p.packed + p.row_bytes;
}

hipError_t launch_paged_weights(int dtype, int n_codewords, const PagedAttendArgs& args, float keep, float* mass, void* workspace, hipStream_t stream) {
  PagedAttendArgs a = args;
  const WeightsPlan plan = plan_of(dtype, n_codewords, a);
  a.slots = plan.slots;
  a.page_groups = a.pool.page_tokens / 8;
  a.page_magic = a.page_groups == 1 ? 0xffffffffu : (uint32_t)((uint64_t(1) << 32) / a.page_groups);
  WeightsArgs x = {};
  unsigned char* at = static_cast<unsigned char*>(workspace);
  const auto take = [&](size_t n) { unsigned char* const p = at; at += n; return p; };
  x.scores = reinterpret_cast<float*>(take(plan.scores));
  x.stats = reinterpret_cast<f32x2*>(take(plan.stats));
  x.heads = reinterpret_cast<int2*>(take(plan.heads));
  x.packed = reinterpret_cast<u32x4*>(take(plan.packed));
  x.rows = reinterpret_cast<WeightsArgs::Row*>(take(plan.row_bytes));
  x.mass = mass; x.keep = keep;
  x.row_cap = plan.rows; x.tiles = (plan.rows + 15) / 16; x.room = (int)plan.room;
  const bool far = (uint64_t)a.pool.rows * a.H * (kGroup / 2) > 0xffffffffull;
  const dim3 grid(plan.blocks, plan.row_tiles);
#define AQUAKV_SCORES(T, N, COLS)                                                                                                    \
  (far ? weights_scores_kernel<T, N, COLS, true><<<grid, ScoreShape<T, N, COLS>::kThreads, 0, stream>>>(a, x)                         \
       : weights_scores_kernel<T, N, COLS, false><<<grid, ScoreShape<T, N, COLS>::kThreads, 0, stream>>>(a, x))
  if (plan.few) {
    AQUAKV_PAGED(dtype, n_codewords, (AQUAKV_SCORES(T, N, 1)));
  } else {
    AQUAKV_PAGED(dtype, n_codewords, (AQUAKV_SCORES(T, N, 2)));
  }
#undef AQUAKV_SCORES
  if (const hipError_t e = hipGetLastError()) return e;
  if (plan.few) {
    weights_from_scores_kernel<<<dim3((unsigned)((plan.room + kChunk - 1) / kChunk * a.H), (unsigned)a.batch), 256, 0, stream>>>(a, x);
    return hipGetLastError();
  }
  const dim3 tiles((unsigned)(x.tiles * a.H), (unsigned)a.batch);
  AQUAKV_PAGED(dtype, n_codewords, (weights_rows_kernel<T, N><<<tiles, 64, 0, stream>>>(a, x)));
  if (const hipError_t e = hipGetLastError()) return e;
  const dim3 tokens((unsigned)((plan.room + kMassTokens - 1) / kMassTokens * a.H), (unsigned)a.batch);
  AQUAKV_PAGED_N(n_codewords, (weights_mass_kernel<N><<<tokens, 64 * kMassWaves, 0, stream>>>(a, x)));
  return hipGetLastError();
}

}  // namespace aquakv
