// Attention over a cache that lives in pages of codes (4 bits and the framework's other widths), read as they are: no row is recovered.
// With the rotation R = H S / sqrt(128) of the quantizer (Sect. 2 of the AQUA-KV paper) a key is R^T (sigma C[codes]), so
//   q . khat = sigma (R q) . C[codes],      sum_t p_t vhat_t = R^T sum_t (p_t sigma_t) C[codes_t]:
// the query is rotated once, the result once, and in between a code is a look-up.  (Uniform backbone: no rotation, (code - zero) step.)
#include "paged_attend.h"

#include <algorithm>

namespace aquakv {
namespace {

using namespace paged;

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
  static constexpr int kWaves = is_rtn(NCW) || COLS == 2 ? 4 : 8;
  static constexpr int kPerSimd = COLS == 2 ? 2 : is_rtn(NCW) ? 3 : sizeof(T) == 4 ? 2 : 4;
  // COLS = 2: a workgroup's waves take pieces of one kv head, one behind the other, and join their results (5 queries of 8 x 9999 tokens, 3 bits: 33.2 us,
  // two waves of two heads each 34.5, every wave its own result 37.6).  With 16 rows they take all heads of the same tokens, whose codes share cache
  // lines: 32 x 16 384 tokens 95.6 us, four waves of two heads joined 99.5, two of four heads 109, one head 113 (one sequence of 131 072: 47, 45, 47, 49).
  static constexpr bool kJoined = COLS == 2;
  static constexpr int kThreads = 64 * kWaves, kSlots = 256 * 4 * kPerSimd;            // threads, waves on the chip
};
template <typename T, int NCW, int COLS, bool FAR>
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
  if constexpr (kJoined) {                                 // workgroups go round the eight chiplets: those of the heads of a piece are eight apart
    const unsigned turn = blockIdx.x >> 3;
    h = turn % a.H;
    item = (turn / a.H * 8 + (blockIdx.x & 7)) * kWaves + wave;
  } else {
    const unsigned unit = blockIdx.x * kWaves + wave;
    h = uniform(unit % a.H);
    item = uniform(unit / a.H);
  }
  const Share share = share_of(a, lane, item);
  if ((kJoined ? item - wave : (int)(blockIdx.x * kWaves / a.H)) >= share.items) return;      // (the whole workgroup is behind the last piece)
  const int b = max(share.b, 0), rep = a.q_heads / a.H;
  const PagedQueries w = paged_queries(a, b);
  const int n_rows = w.n * rep, row0 = blockIdx.y * kRows;
  const bool idle = share.b < 0 || row0 >= n_rows;
  // the tokens of this piece
  const int first_limit = uniform(w.len - w.count + row0 / rep), last_limit = uniform(w.len - w.count + min(row0 + kRows - 1, n_rows - 1) / rep);
  const TokenRange range = piece_range(share.piece, share.tiles, kTile, idle ? 0 : last_limit + 1);
  const int t_begin = range.begin, t_end = range.end;
  const bool any = t_begin < t_end;
  typename C::Column col[COLS];
  typename C::template Query<T> asked[COLS] = {};
  if (!idle) {
#pragma unroll
    for (int i = 0; i < COLS; ++i) {                       // (rows that are not there: the last one again, which sees nothing)
      const int row = row0 + 16 * i + m, there = min(row, n_rows - 1), qi = there / rep, qh = h * rep + there % rep;
      col[i].limit = row < n_rows ? w.len - w.count + qi : -1;
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
    float lift[COLS];                                      // power of two of the largest scale of the lane's tokens that the row sees
    if constexpr (COLS > 1) {
#pragma unroll
      for (int i = 0; i < COLS; ++i) lift[i] = C::lift_of(vs);
    }
    if (masked) {
      asm volatile("");                                    // (a branch, not selects that every tile would pay for)
#pragma unroll
      for (int i = 0; i < COLS; ++i) {
        const int seen = min(col[i].limit + 1 - (t + 8 * g), held);
#pragma unroll
        for (int e = 0; e < 8; ++e) p[i][e] = e < seen ? p[i][e] : -INFINITY;
        u32x4 own[C::kHalves];
#pragma unroll
        for (int k = 0; k < C::kHalves; ++k) {
          own[k] = vs[k];
          C::keep_first(own[k], seen);
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
    int seen[COLS];
#pragma unroll
    for (int i = 0; i < COLS; ++i) seen[i] = min(col[i].limit + 1 - (t + 8 * g), held);
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
  if (a.heads != nullptr && !idle && share.piece == 0 && h == 0 && blockIdx.y == 0 && lane == 0) a.heads[b] = int2{result, results};
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

// results from, from + by, ... below `pieces` of the row at `at` (results `step` rows apart): four coordinates of the sum, the reference, the sum of weights
struct Joined { f32x4 x; float ref, sum; };
__device__ __forceinline__ Joined join_results(const PagedAttendArgs& a, int64_t at, int64_t step, int from, int by, int pieces, int l) {
  constexpr int kAhead = 4;
  Joined j = {f32x4{0.f, 0.f, 0.f, 0.f}, -3.0e38f, 0.f};
  for (int i0 = from; i0 < pieces; i0 += kAhead * by) {
    f32x2 st[kAhead];
    f32x4 p[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int i = i0 + u * by;
      st[u] = f32x2{-3.0e38f, 0.f};
      p[u] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (i < pieces) {
        st[u] = *reinterpret_cast<const f32x2*>(a.stats + 2 * (at + i * step));
        p[u] = *reinterpret_cast<const f32x4*>(a.part + (at + i * step) * kGroup + 4 * l);
      }
    }
    float top = j.ref;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) top = fmaxf(top, st[u].x);
    const float keep = __builtin_amdgcn_exp2f(j.ref - top);
    j.x *= keep;
    j.sum *= keep;
    j.ref = top;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const float by2 = __builtin_amdgcn_exp2f(st[u].x - top);
      j.x += p[u] * by2;
      j.sum += st[u].y * by2;
    }
  }
  return j;
}
// a joined row, 16 coordinates on each of eight lanes as in the stand-alone inverse -> out
template <typename T, bool RTN> __device__ __forceinline__ void finish_joined(const PagedAttendArgs& a, const float* row, int lane, int h, int64_t to) {
  const int q = group_pos<16>(lane);
  float v[16];
  load_f32(row + 16 * q, v);
  if constexpr (!RTN) {
    float sf[16];
    load_signs(a.signs_v, h, q, sf);
    const float norm = kRsqrtG * Rot<false>::sign(q);
#pragma unroll
    for (int r = 0; r < 16; ++r) v[r] *= norm;
    Rot<false>::iwht(v, q);
#pragma unroll
    for (int r = 0; r < 16; ++r) v[r] *= sf[r];
  }
  Storage<T>::template store<false>(static_cast<T*>(a.out) + to * kGroup, q, v);
}
// out of one row from the pieces of its sequence: sum_i 2^(ref_i - top) part_i / sum_i 2^(ref_i - top) sum_i.
// blockIdx = (query * q_heads + query head, sequence); threads of 32 take a piece each, 4 coordinates a thread, and go on by as many pieces as there
// are such groups: 8, or 32 where there are many pieces.  All partial results of a round are requested together, ahead of the sequence's numbers.
// A chain of waits of 3 to 5 us whatever its size (24 sequences in some 19 pieces each: 4.8 us) but for one long sequence's (512 pieces of 64 heads, 17 MB: 8.8 us).
template <typename T, bool RTN, int THREADS>
__global__ __launch_bounds__(THREADS) void paged_merge_kernel(const PagedAttendArgs a) {
  constexpr int kClasses = THREADS / 32;
  __shared__ __align__(16) float red[kClasses][kGroup];
  __shared__ float refs[kClasses], sums[kClasses];
  __shared__ __align__(16) float row[kGroup];
  const int b = blockIdx.y, qi = blockIdx.x / a.q_heads, qh = blockIdx.x % a.q_heads, h = qh / (a.q_heads / a.H);
  const int2 head = a.heads[b];
  const int pieces = uniform(head.y);
  if (pieces == 1) return;
  const PagedQueries w = paged_queries(a, b);
  if (qi >= w.n) return;
  const int k = threadIdx.x >> 5, l = threadIdx.x & 31;
  const int64_t step = (int64_t)a.max_queries * a.q_heads, at = uniform(head.x) * step + (int64_t)qi * a.q_heads + qh;
  const Joined j = join_results(a, at, step, k, kClasses, pieces, l);
  *reinterpret_cast<f32x4*>(&red[k][4 * l]) = j.x;
  if (l == 0) { refs[k] = j.ref; sums[k] = j.sum; }
  __syncthreads();
  if (threadIdx.x < kGroup) {                              // a thread per coordinate
    float top = refs[0];
#pragma unroll
    for (int i = 1; i < kClasses; ++i) top = fmaxf(top, refs[i]);
    float total = 0.f, value = 0.f;
#pragma unroll
    for (int i = 0; i < kClasses; ++i) {
      const float by = __builtin_amdgcn_exp2f(refs[i] - top);
      total += sums[i] * by;
      value = __fmaf_rn(red[i][threadIdx.x], by, value);
    }
    row[threadIdx.x] = value * (total == 0.f ? 0.f : 1.0f / total);
  }
  __syncthreads();
  if (threadIdx.x >= 8) return;
  finish_joined<T, RTN>(a, row, threadIdx.x, h, (w.first + qi) * a.q_heads + qh);
}
// The same for many rows of few pieces: eight rows a workgroup, 32 threads each, so that the way back takes a whole wave (1000 queries of 32 heads over 1000
// tokens: 50 us, a row a workgroup 77; 512 over 6000: 92, 104; 130 sequences of 700 tokens 33, 36; where rows have some 20 pieces the loop over them
// is the longer chain: 24 x 3000 tokens 28.8, 27.0).
template <typename T, bool RTN>
__global__ __launch_bounds__(256) void paged_merge_rows_kernel(const PagedAttendArgs a) {
  __shared__ __align__(16) float rows[8][kGroup];
  const int b = blockIdx.y, first = 8 * blockIdx.x;         // rows of the sequence: query * q_heads + query head
  const int2 head = a.heads[b];
  const int pieces = uniform(head.y);
  if (pieces == 1) return;
  const PagedQueries w = paged_queries(a, b);
  const int n_rows = w.n * a.q_heads;
  if (first >= n_rows) return;
  const int k = threadIdx.x >> 5, l = threadIdx.x & 31;
  const int64_t step = (int64_t)a.max_queries * a.q_heads, at = uniform(head.x) * step + min(first + k, n_rows - 1);
  const Joined j = join_results(a, at, step, 0, 1, pieces, l);
  *reinterpret_cast<f32x4*>(&rows[k][4 * l]) = j.x * (j.sum == 0.f ? 0.f : 1.0f / j.sum);
  __syncthreads();
  const int r = first + (threadIdx.x >> 3);
  if (threadIdx.x < 64) {                                  // (rows that are not there stay for the exchanges of lanes)
    const int there = min(r, n_rows - 1);
    finish_joined<T, RTN>(a, rows[there - first], threadIdx.x & 7, there % a.q_heads / (a.q_heads / a.H), w.first * a.q_heads + there);
  }
}

// How a launch is laid out, from sizes alone (lengths and counts of queries are on the device): by max_queries, whatever the sequences have.  So single queries
// beside a chunk are walked by one workgroup a kv head each, as a block of 256 rows is: 31 over 16 384 tokens and a chunk of 512, 32 heads, 2.1 ms, in a call of
// their own 94 us, the chunk by itself 99.
struct PagedPlan { unsigned blocks, row_tiles; int slots, row_blocks; int64_t items; bool two, merge, many, by_rows; };
// Results of a sequence beyond which the merge has 1024 threads a row, of 256 (one query of 131 072 tokens 41.0 us, for 45.0; beyond 8: 32 x 4000 tokens
// 37.4 for 34.4).
constexpr int kManyPieces = 64;
// Rows of a kv head up to which waves of 32 take them in turn (8 x 9999 tokens, 3 bits: 68 rows 108 us, in tiles of 256 rows 131; 128 rows 93, 135; 32 x 4000:
// 167, 167 and 150, 170; one sequence of 12 288: 35, 31 and 31, 35; 192 rows of 8 x 9999: 230, 136).
constexpr int kFewRows = 128;
template <typename T, int NCW> PagedPlan paged_plan(int64_t batch, int64_t table_pages, int64_t page_tokens, int64_t max_queries, int64_t q_heads, int64_t H) {
  PagedPlan p = {};
  const int64_t rows = std::max<int64_t>(max_queries, 1) * (q_heads / H), most = (table_pages * page_tokens + kTile - 1) / kTile;      // tiles of a sequence
  if (sizeof(T) == 2 && rows > kFewRows) {                 // workgroups of 256 rows, one a CU: the tokens in pieces if there are too few of them
    p.row_blocks = (int)((rows + kTileRows - 1) / kTileRows);
    // ... of 4 tiles of 64 at least, of 2 where there is one block of rows and so little to join (180 rows over 700 tokens: 28.0 us, 22.2; 160 over 6000: 34.3, 31.5;
    // 1200 rows over 300: 23.3, 26.2)
    p.slots = (int)std::max<int64_t>(std::min(256 / std::max<int64_t>(batch * H * p.row_blocks, 1), most / (p.row_blocks == 1 ? 4 : 8)), 1);
    p.items = batch * p.slots;
    p.merge = p.slots > 1;
    p.by_rows = p.slots <= 16;
    p.many = p.slots > kManyPieces;
    return p;
  }
  // 9 to 16 rows fill one column of a wave, but two columns take as long and join their results (16 rows of 8 x 9999 tokens, 3 bits: 37.3 us, in one column
  // 39.7; of one sequence of 12 288: 18.9, 29.8; of 32 x 4000 46.1, 44.8); 8 rows do not (one sequence of 131 072: 49.0, 41.9; 32 x 16 384: 138, 101; 8 x 9999 31.3,
  // 30.4; but one of 16 384 18.0, 19.8).
  p.two = sizeof(T) == 2 && rows > 8;
  const int per_wave = p.two ? 32 : 16, waves = p.two ? Shape<T, NCW, 2>::kWaves : Shape<T, NCW, 1>::kWaves;
  p.row_tiles = (unsigned)((rows + per_wave - 1) / per_wave);
  // As many pieces as make all waves that the chip holds (32 x 16 384 tokens: 95.7 us, half as many 111, twice as many 99; 5 queries of 8 x 9999 37.7, 42.8,
  // 50.7); the kernel makes fewer of short ones.
  p.slots = (int)std::max<int64_t>((p.two ? Shape<T, NCW, 2>::kSlots : Shape<T, NCW, 1>::kSlots) / (H * p.row_tiles), 1);
  const int64_t pieces = std::min(batch * std::max<int64_t>(most, 1), std::max<int64_t>(p.slots - batch, std::max(p.slots / 2, 1)) + batch);
  if (p.two) {                                             // (a workgroup has results of as many sequences as it has pieces of)
    const int64_t groups = (pieces + waves - 1) / waves;
    p.blocks = (unsigned)((groups + 7) / 8 * 8 * H);
    p.items = groups + batch;
    p.merge = groups > 1;
  } else {
    p.blocks = (unsigned)((pieces * H + waves - 1) / waves);
    p.items = pieces;
    p.merge = most > 1;
  }
  p.many = p.items > kManyPieces * batch;
  p.by_rows = p.items <= 8 * batch && batch * max_queries * q_heads >= 512;
  return p;
}

}  // namespace

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

static PagedPlan plan_of(int dtype, int n_codewords, const PagedAttendArgs& a) {
  PagedPlan p = {};
  AQUAKV_PAGED(dtype, n_codewords, (p = paged_plan<T, N>(a.batch, a.table_pages, a.pool.page_tokens, a.max_queries, a.q_heads, a.H)));
  return p;
}

size_t paged_attend_workspace_bytes(int dtype, int n_codewords, const PagedAttendArgs& a) {
  const PagedPlan p = plan_of(dtype, n_codewords, a);
  if (!p.merge) return 0;
  return (size_t)p.items * a.max_queries * a.q_heads * (kGroup + 2) * sizeof(float) + (size_t)a.batch * sizeof(int2);
}

hipError_t launch_paged_attend(int dtype, int n_codewords, const PagedAttendArgs& args, void* workspace, hipStream_t stream) {
  PagedAttendArgs a = args;
  const PagedPlan plan = plan_of(dtype, n_codewords, a);
  a.slots = plan.slots;
  a.row_blocks = plan.row_blocks;
  a.part = static_cast<float*>(workspace);
  a.stats = a.part + plan.items * a.max_queries * a.q_heads * kGroup;
  a.heads = plan.merge ? reinterpret_cast<int2*>(a.stats + plan.items * a.max_queries * a.q_heads * 2) : nullptr;
  a.page_groups = a.pool.page_tokens / 8;
  a.page_magic = a.page_groups == 1 ? 0xffffffffu : (uint32_t)((uint64_t(1) << 32) / a.page_groups);
  if (plan.row_blocks != 0) {
    if (const hipError_t e = launch_paged_tiles(n_codewords, a, stream)) return e;
  } else {
    const bool far = (uint64_t)a.pool.rows * a.H * (kGroup / 2) > 0xffffffffull;      // (codes take half a byte per value at most)
    const dim3 blocks(plan.blocks, plan.row_tiles);
#define AQUAKV_ATTEND(T, N, COLS)                                                                                        \
  (far ? paged_attend_kernel<T, N, COLS, true><<<blocks, Shape<T, N, COLS>::kThreads, 0, stream>>>(a)                     \
       : paged_attend_kernel<T, N, COLS, false><<<blocks, Shape<T, N, COLS>::kThreads, 0, stream>>>(a))
    if (plan.two) {
      typedef bf16_t T;
      AQUAKV_PAGED_N(n_codewords, (AQUAKV_ATTEND(T, N, 2)));
    } else {
      AQUAKV_PAGED(dtype, n_codewords, (AQUAKV_ATTEND(T, N, 1)));
    }
#undef AQUAKV_ATTEND
    if (const hipError_t e = hipGetLastError()) return e;
  }
  if (!plan.merge) return hipSuccess;
  const dim3 grid((unsigned)(a.max_queries * a.q_heads), (unsigned)a.batch);
  const bool rtn = is_rtn(n_codewords);
  const dim3 by_rows((unsigned)((a.max_queries * a.q_heads + 7) / 8), (unsigned)a.batch);
#define AQUAKV_MERGE(T, RTN)                                                                                  \
  (plan.by_rows ? paged_merge_rows_kernel<T, RTN><<<by_rows, 256, 0, stream>>>(a)                              \
   : plan.many ? paged_merge_kernel<T, RTN, 1024><<<grid, 1024, 0, stream>>>(a)                                  \
             : paged_merge_kernel<T, RTN, 256><<<grid, 256, 0, stream>>>(a))
  if (dtype == kBF16) { if (rtn) AQUAKV_MERGE(bf16_t, true); else AQUAKV_MERGE(bf16_t, false); }
  else { if (rtn) AQUAKV_MERGE(float, true); else AQUAKV_MERGE(float, false); }
#undef AQUAKV_MERGE
  return hipGetLastError();
}

}  // namespace aquakv
