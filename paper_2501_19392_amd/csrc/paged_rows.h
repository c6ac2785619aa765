// The kernel of attention over pages for few rows: what paged_attend.hip and, for trees of drafted tokens, paged_tree.hip build.
#pragma once
#include "paged_attend.h"

namespace aquakv {
namespace paged {

// One wave takes `tiles` tiles of 32 tokens of one kv head for up to 16 rows (query x query head of the kv head): soft-max in one pass with a
// running reference, fp16 matrix instructions (16x16x32) with fp32 sums.  Lane l = 16 g + m:
//   scores   S^T = K Q^T, two products of 16 tokens: A holds token 8 (m / 4) + m % 4 (+ 4 in the second), so that a lane gets the scores of
//            tokens 8 g ... 8 g + 7 for row m, which is what the second product wants of it as its B operand, with no exchange between lanes;
//   values   O^T = V^T P: A holds 8 tokens of one coordinate; a look-up gives two neighbouring coordinates, two permutes pair them up by
//            token.  The 32 coordinates a lane ends with are consecutive, as the inverse transform wants them.
// COLS = 2: 32 rows, on twice the registers; a tile's codes become operands once for both.
// No tile is staged: a wave reads its codes with wide loads a tile ahead and turns them into operands in registers, by a look-up (one permute for the
// address, one LDS read, no bank conflicts) for two coordinates.  Why one wave a piece and not a workgroup: nothing is shared but the grid, and no wave
// waits for another.
//
// Bound by memory for long sequences: 32 x 16 384 tokens, 4 query heads a kv head, 88 us in the kernel, 4.6 TB/s of codes and scales (a copy reaches 5.1),
// vector pipes busy in 60 % of the cycles.  Few tokens: by the chain at its start (lengths, pages, codes, grid, rotated query: 3 us to
// the first score) and the second launch, 4 us: one sequence of 700 tokens 11.1 us a call.  Many rows (8 x 9999 tokens, 5 queries, 3 bits: 33 us): by the vector
// pipes, 54 % busy, and the waits between a tile's two products at two waves a SIMD.
// Times of these three are of calls whose inputs change; those beside the rules below, of the same call again and again in a captured graph, whose codes may stay in
// the caches (one sequence of 131 072 tokens, 8 rows a kv head: 46.4 us with other inputs each time, 41.9 with the same).  All of 8 kv heads.
// Waves of a workgroup, which share the copies of the grid, and waves per SIMD: with 128 registers four fit (two workgroups a CU, which is what LDS has
// room for with 256 points); uniform codes need more for the two halves' scales, and no LDS to speak of; fp32 layers hold everything twice.
template <typename T, int NCW, int COLS> struct Shape {
  static constexpr int kWaves = is_rtn(NCW) || COLS >= 2 ? 4 : 8;
  static constexpr int kPerSimd = COLS >= 2 ? 2 : is_rtn(NCW) ? 3 : sizeof(T) == 4 ? 2 : 4;
  // COLS = 2: a workgroup's waves take pieces of one kv head, one behind the other, and join their results (5 queries of 8 x 9999 tokens, 3 bits: 33.2 us,
  // two waves of two heads each 34.5, every wave its own result 37.6).  With 16 rows they take all heads of the same tokens, whose codes share cache
  // lines: 32 x 16 384 tokens 95.6 us, four waves of two heads joined 99.5, two of four heads 109, one head 113 (one sequence of 131 072: 47, 45, 47, 49).
  static constexpr bool kJoined = COLS >= 2;
  static constexpr int kThreads = 64 * kWaves, kSlots = 256 * 4 * kPerSimd;            // threads, waves on the chip
};
template <typename T, int NCW, int COLS, bool FAR, bool TREE>
__global__ __launch_bounds__((Shape<T, NCW, COLS>::kThreads)) __attribute__((amdgpu_waves_per_eu((Shape<T, NCW, COLS>::kPerSimd)))) void
paged_attend_kernel(const PagedAttendArgs a) {
  constexpr int kWaves = Shape<T, NCW, COLS>::kWaves, kRows = 16 * COLS;
  constexpr int kTerms = sizeof(T) == 2 ? 1 : 2;
  constexpr bool kRtn = is_rtn(NCW);
  typedef Codes<NCW, kTerms> C;
  constexpr bool kJoined = Shape<T, NCW, COLS>::kJoined;
  constexpr int kPiece = 16 * (kGroup + 2) * 4;            // bytes of 16 rows' sums, references and sums of weights
  constexpr int kJoinBytes = kJoined ? (kWaves - 1) * COLS * kPiece : 0, kTable = kJoinBytes > C::kTableBytes ? kJoinBytes : C::kTableBytes;
  __shared__ __align__(256) unsigned char lds[kTable + kWaves * C::kScaleBytes];
  const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  unsigned char* const scale_lds = lds + kTable + wave * C::kScaleBytes;

  // What is waited for at the start is a chain (lengths, then the piece's pages, then its codes); all else is requested beside it.
  const typename C::Points points = C::request_points(a.codebook, lane);
  // which rows, kv head and piece of a sequence
  int h, item;
  unsigned row_tile = blockIdx.y;
  if constexpr (kJoined) {                                 // workgroups go round the eight chiplets: those of the heads of a piece are eight apart
    const unsigned turn = blockIdx.x >> 3;
    unsigned group = turn / a.H * 8 + (blockIdx.x & 7);
    h = turn % a.H;
    if constexpr (TREE) {
      // Row tiles of a piece come to the same CU, one behind the other, where the pieces fill all chiplets alike (4 tiles, 32 x 8000 tokens: 246 us, else 262);
      // otherwise they go round the chiplets with the pieces (3 tiles, 21 groups of pieces: 187 us, else 297, as five chiplets would have 72 workgroups, for 64 that
      // run at once).
      if (a.rows_apart) {
        row_tile = group % a.row_tiles;
        group /= a.row_tiles;
      }
    }
    item = group * kWaves + wave;
  } else {
    const unsigned unit = blockIdx.x * kWaves + wave;
    h = uniform(unit % a.H);
    item = uniform(unit / a.H);
  }
  const Share share = share_of(a, lane, item);
  if ((kJoined ? item - wave : (int)(blockIdx.x * kWaves / a.H)) >= share.items) return;      // (the whole workgroup is behind the last piece)
  const int b = max(share.b, 0), rep = a.q_heads / a.H;
  const PagedQueries w = paged_queries(a, b);
  const int n_rows = w.n * rep, row0 = row_tile * kRows;
  const bool idle = share.b < 0 || row0 >= n_rows;
  // the tokens of this piece
  const int past = w.len - w.count;                        // tokens ahead of the queries' own
  const int first_limit = TREE ? past - 1 : uniform(past + row0 / rep);
  const int last_limit = TREE ? w.len - 1 : uniform(past + min(row0 + kRows - 1, n_rows - 1) / rep);
  const TokenRange range = piece_range(share.piece, share.tiles, kTile, idle ? 0 : last_limit + 1);
  const int t_begin = range.begin, t_end = range.end;
  const bool any = t_begin < t_end;
  typename C::Column col[COLS];
  typename C::template Query<T> asked[COLS] = {};
  if (!idle) {
#pragma unroll
    for (int i = 0; i < COLS; ++i) {                       // (rows that are not there: the last one again, which sees nothing)
      const int row = row0 + 16 * i + m, there = min(row, n_rows - 1), qi = there / rep, qh = h * rep + there % rep;
      if constexpr (TREE) col[i].limit = row < n_rows ? qi : -1;
      else col[i].limit = row < n_rows ? past + qi : -1;
      asked[i] = C::template request_query<T>(static_cast<const T*>(a.q) + (w.first + qi) * a.q_stride + qh * kGroup, a.signs_k, h, g);
    }
  }
  Rows r0 = {}, r1 = {};
  typename C::Keys k = {}, next = {};
  typename C::Values v = {};
  if (any) {
    r0 = rows_of(a, b, t_begin);
    r1 = rows_of(a, b, t_begin + kTile);
    k = C::template request_keys<FAR>(a, r0, h, lane);
    v = C::template request_values<FAR>(a, r0, h, lane);
  }
  const int c_exp = C::template stage<kWaves>(points, lds, lane, wave);
  __syncthreads();
  if (!kJoined && idle) return;

  // ---- the rows' queries: rotated, scaled to fp16's range
#pragma unroll
  for (int i = 0; i < COLS; ++i) {
    if (idle) break;
    float x[32];
    C::template rotate_query<T>(asked[i], lane, x);
    const float by = a.scale * 1.4426950408889634f * (kRtn ? 1.0f : kRsqrtG);
    float top = 0.f;
#pragma unroll
    for (int r = 0; r < 32; ++r) top = fmaxf(top, fabsf(x[r]));
    const int e = max(__builtin_amdgcn_frexp_expf(column_max(top) * fabsf(by)), -100);
    col[i].f = __builtin_ldexpf(1.0f, min(e - kQueryExp + (kRtn ? C::kFieldExp : c_exp), 126));
    const float scaled = __builtin_ldexpf(by, kQueryExp - e);
#pragma unroll
    for (int r = 0; r < 32; ++r) x[r] *= scaled;
    C::pack_query(x, col[i].q, col[i].qsum);
#pragma unroll
    for (int j = 0; j < 8; ++j) col[i].o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < C::kHalves; ++j) col[i].oz[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    col[i].ref = -3.0e38f;
    col[i].sum = 0.f;
  }

  const auto tile = [&](const typename C::Keys& x, const typename C::Values& xv, int t, unsigned there) {
    // scales of the tile's 32 tokens to the lanes that need them
    asm volatile("" ::: "memory");                         // (a wave's LDS accesses stay in order)
    C::put_scales(x, scale_lds, lane);
    asm volatile("" ::: "memory");
    f32x4 s[COLS][C::kHalves][2] = {};                     // [column][half][product]
#pragma unroll
    for (int p = 0; p < 2; ++p) C::scores(x, p, lds, lane, col, s);
    __builtin_amdgcn_sched_barrier(0);
    float p[COLS][8];
#pragma unroll
    for (int i = 0; i < COLS; ++i) C::scaled(s[i], scale_lds, g, col[i].qsum, p[i]);
    u32x4 vs[C::kHalves];
#pragma unroll
    for (int k = 0; k < C::kHalves; ++k) vs[k] = C::value_scales(scale_lds, k, g);
    const int held = (there >> g) & 1 ? w.len - (t + 8 * g) : 0;           // so many of the lane's eight tokens are there: the others hold anything
    const bool masked = t + kTile - 1 > first_limit || t + kTile > t_end || there != 15u;      // (t_end: of this piece, whole tiles but for the last)
    typedef SeenOf<TREE> Seen;
    Seen seen[COLS];                                       // which of the lane's eight tokens the row sees
    const auto look = [&](int i) {
      if constexpr (TREE) seen[i].bits = col[i].limit < 0 ? 0u : tree_bits(a, w.first + col[i].limit, t + 8 * g - past) & first_bits(held);
      else seen[i].n = min(col[i].limit + 1 - (t + 8 * g), held);
    };
    float lift[COLS];                                      // power of two of the largest scale of the lane's tokens that the row sees
    if constexpr (COLS > 1) {
#pragma unroll
      for (int i = 0; i < COLS; ++i) lift[i] = C::lift_of(vs);
    }
    if (masked) {
      asm volatile("");                                    // (a branch, not selects that every tile would pay for)
#pragma unroll
      for (int i = 0; i < COLS; ++i) {
        look(i);
#pragma unroll
        for (int e = 0; e < 8; ++e) p[i][e] = seen[i].has(e) ? p[i][e] : -INFINITY;
        u32x4 own[C::kHalves];
#pragma unroll
        for (int k = 0; k < C::kHalves; ++k) {
          own[k] = vs[k];
          seen[i].keep(own[k]);
          if constexpr (COLS == 1) vs[k] = own[k];
        }
        if constexpr (COLS > 1) lift[i] = C::lift_of(own);
      }
    }
    if constexpr (COLS == 1) lift[0] = C::lift_of(vs);
    // The reference follows where the largest weight that the scores allow is too large: such weights become 2^kStartExp.
    float top[COLS];
    bool high = false;
#pragma unroll
    for (int i = 0; i < COLS; ++i) {
      top[i] = p[i][0];
#pragma unroll
      for (int e = 1; e < 8; ++e) top[i] = fmaxf(top[i], p[i][e]);
      high |= __fmaf_rn(top[i], col[i].f, lift[i] - col[i].ref) > kTopExp;
    }
    if (__builtin_amdgcn_ballot_w64(high) != 0) {
#pragma unroll
      for (int i = 0; i < COLS; ++i) {
        const float moved = fmaxf(col[i].ref, column_max(__fmaf_rn(top[i], col[i].f, lift[i])) - kStartExp);
        const float by = __builtin_amdgcn_exp2f(col[i].ref - moved);
        col[i].ref = moved;
        col[i].sum *= by;
#pragma unroll
        for (int j = 0; j < 8; ++j) col[i].o[j] *= by;
        if constexpr (kRtn) { col[i].oz[0] *= by; col[i].oz[1] *= by; }
      }
    }
#pragma unroll
    for (int i = 0; i < COLS; ++i) {
#pragma unroll
      for (int e = 0; e < 8; ++e) p[i][e] = __builtin_amdgcn_exp2f(__fmaf_rn(p[i][e], col[i].f, -col[i].ref));
      col[i].sum += sum_of(p[i]);
    }
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (!TREE) {                                 // (worked out anew: no registers for them in between)
#pragma unroll
      for (int i = 0; i < COLS; ++i) look(i);
    }
    C::values(xv, scale_lds, held, masked, seen, p, vs, lds, lane, col);
  };
  // Keys are requested a tile ahead, values behind the tile that takes their registers, the rows they are in two tiles ahead.
#pragma unroll 1
  for (int t = t_begin; t < t_end; t += kTile) {
    const bool more = t + kTile < t_end;
    if (more) next = C::template request_keys<FAR>(a, r1, h, lane);
    const unsigned there = there_of(r0);
    const Rows r2 = rows_of(a, b, t + 2 * kTile);
    tile(k, v, t, there);
    if (more) v = C::template request_values<FAR>(a, r1, h, lane);
    k = next;
    r0 = r1;
    r1 = r2;
  }

  // Results of a sequence that others than this workgroup (wave) have: their number, and which this one's is.
  int results = share.pieces, result = item;
  int others = 0;                                          // waves behind this one whose results it takes
  if constexpr (kJoined) {
    const int first = item - share.piece, group = (item - wave) / kWaves;
    results = (first + share.pieces - 1) / kWaves - first / kWaves + 1;
    result = group + b;                                    // (two sequences that share a workgroup are neighbours)
    others = min(kWaves - wave, share.pieces - share.piece) - 1;
  }
  if (a.heads != nullptr && !idle && share.piece == 0 && h == 0 && row_tile == 0 && lane == 0) a.heads[b] = int2{result, results};
  // (worked out anew: lane and row numbers are not worth registers in the loop)
  int again = lane;
  asm volatile("" : "+v"(again));
  const auto place = [&](int w, int i) { return reinterpret_cast<f32x4*>(lds + ((w - 1) * COLS + i) * kPiece); };
  if constexpr (kJoined) {
    // the first wave of each sequence takes the others' sums, which go where the grid was
    const bool gives = wave != 0 && share.piece != 0;
    __syncthreads();
    if (gives && !idle) {
#pragma unroll
      for (int i = 0; i < COLS; ++i) {
        const float sum = column_sum(col[i].sum);
        float x[32];
        C::result(col[i], kRtn ? C::kFieldExp : c_exp, x);
        f32x4* const to = place(wave, i);
#pragma unroll
        for (int r = 0; r < 8; ++r) to[64 * r + again] = f32x4{x[4 * r], x[4 * r + 1], x[4 * r + 2], x[4 * r + 3]};
        if (again < 16) reinterpret_cast<f32x2*>(to + 512)[again] = f32x2{col[i].ref, sum};
      }
    }
    __syncthreads();
    if (gives || idle) return;
  }
  // ---- the lane's 32 coordinates of the row
#pragma unroll
  for (int i = 0; i < COLS; ++i) {
    const int row = row0 + 16 * i + (again & 15), qi = row / rep, qh = h * rep + row % rep;
    float x[32], ref = col[i].ref, sum = column_sum(col[i].sum);
    C::result(col[i], kRtn ? C::kFieldExp : c_exp, x);
    if constexpr (kJoined) {
#pragma unroll 1
      for (int n = 1; n <= others; ++n) {
        const f32x4* const from = place(wave + n, i);
        const f32x2 st = reinterpret_cast<const f32x2*>(from + 512)[again & 15];
        const float top = fmaxf(ref, st.x), keep = __builtin_amdgcn_exp2f(ref - top), by = __builtin_amdgcn_exp2f(st.x - top);
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          const f32x4 y = from[64 * r + again];
#pragma unroll
          for (int e = 0; e < 4; ++e) x[4 * r + e] = __fmaf_rn(y[e], by, x[4 * r + e] * keep);
        }
        sum = __fmaf_rn(st.y, by, sum * keep);
        ref = top;
      }
    }
    if (results == 1) {
      finish<T, NCW>(a, x, sum, h, again, row < n_rows, w.first + qi, qh);
    } else if (row < n_rows) {
      const int64_t at = ((int64_t)result * a.max_queries + qi) * a.q_heads + qh;
      float* const part = a.part + at * kGroup;
#pragma unroll
      for (int r = 0; r < 8; ++r)
        *reinterpret_cast<f32x4*>(part + C::coordinate(again >> 4, 4 * r)) = f32x4{x[4 * r], x[4 * r + 1], x[4 * r + 2], x[4 * r + 3]};
      if (again < 16) *reinterpret_cast<f32x2*>(a.stats + 2 * at) = f32x2{ref, sum};
    }
  }
}

#define AQUAKV_PAGED(DT, NCW, CALL)                                            \
  do {                                                                         \
    if ((DT) == kBF16) { typedef bf16_t T; AQUAKV_PAGED_N(NCW, CALL); }        \
    else { typedef float T; AQUAKV_PAGED_N(NCW, CALL); }                       \
  } while (0)
#define AQUAKV_PAGED_N(NCW, CALL)                                              \
  do {                                                                         \
    if ((NCW) == kRtn2) { constexpr int N = kRtn2; CALL; }                     \
    else if ((NCW) == kRtn4) { constexpr int N = kRtn4; CALL; }                \
    else if ((NCW) == 16) { constexpr int N = 16; CALL; }                      \
    else if ((NCW) == 64) { constexpr int N = 64; CALL; }                      \
    else { constexpr int N = 256; CALL; }                                      \
  } while (0)

template <bool TREE> hipError_t launch_rows(int dtype, int n_codewords, int cols, dim3 blocks, const PagedAttendArgs& a, hipStream_t stream) {
  const bool far = (uint64_t)a.pool.rows * a.H * (kGroup / 2) > 0xffffffffull;      // (codes take half a byte per value at most)
#define AQUAKV_ATTEND(T, N, COLS)                                                                                             \
  (far ? paged_attend_kernel<T, N, COLS, true, TREE><<<blocks, Shape<T, N, COLS>::kThreads, 0, stream>>>(a)                    \
       : paged_attend_kernel<T, N, COLS, false, TREE><<<blocks, Shape<T, N, COLS>::kThreads, 0, stream>>>(a))
  if (cols == 2) {
    typedef bf16_t T;
    AQUAKV_PAGED_N(n_codewords, (AQUAKV_ATTEND(T, N, 2)));
  } else if (cols == 3) {                                  // (trees, grids)
    if constexpr (TREE) {
      typedef bf16_t T;
      if (n_codewords == 16) AQUAKV_ATTEND(T, 16, 3);
      else if (n_codewords == 64) AQUAKV_ATTEND(T, 64, 3);
      else AQUAKV_ATTEND(T, 256, 3);
    }
  } else {
    AQUAKV_PAGED(dtype, n_codewords, (AQUAKV_ATTEND(T, N, 1)));
  }
#undef AQUAKV_ATTEND
  return hipGetLastError();
}

}  // namespace paged
}  // namespace aquakv
