// Attention over a cache that lives in pages of codes (4 bits and the framework's other widths), read as they are: no row is recovered.
// With the rotation R = H S / sqrt(128) of the quantizer (Sect. 2 of the AQUA-KV paper) a key is R^T (sigma C[codes]), so
//   q . khat = sigma (R q) . C[codes],      sum_t p_t vhat_t = R^T sum_t (p_t sigma_t) C[codes_t]:
// the query is rotated once, the result once, and in between a code is a look-up.  (Uniform backbone: no rotation, (code - zero) step.)
#include "paged_rows.h"

#include <algorithm>

namespace aquakv {
namespace {

using namespace paged;

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
struct PagedPlan { unsigned blocks, row_tiles, rows_apart; int slots, row_blocks; int64_t items, results; int cols; bool merge, many, by_rows; };      // results: kept for the merge
// Results of a sequence beyond which the merge has 1024 threads a row, of 256 (one query of 131 072 tokens 41.0 us, for 45.0; beyond 8: 32 x 4000 tokens
// 37.4 for 34.4).
constexpr int kManyPieces = 64;
// Rows of a kv head up to which waves of 32 take them in turn (8 x 9999 tokens, 3 bits: 68 rows 108 us, in tiles of 256 rows 131; 128 rows 93, 135; 32 x 4000:
// 167, 167 and 150, 170; one sequence of 12 288: 35, 31 and 31, 35; 192 rows of 8 x 9999: 230, 136).
constexpr int kFewRows = 128;
// Trees: columns of 16 rows that a wave has, by the rows of a kv head and the tiles of all sequences and heads.  Three take the codes to operands once where two would do it
// twice, on all registers there are (uniform codes need more than there are for two waves a SIMD: 48 rows 137 us, with three columns and one wave 152): 36 rows of 32 x 8000 tokens (256 points) 83 us, with two 119; 80 rows 149, 187; 144 rows 215, 436; 64
// rows, two tiles either way, 148, 122.  Where a wave has few tiles, more waves are better: 36 rows of 16 000 tokens 23.9, 22.5; of 2000 16.4, 14.6.
int tree_columns(int64_t rows, bool rtn, int64_t tiles) {
  if (rows <= 8) return 1;
  return !rtn && tiles >= 8192 && (rows + 47) / 48 < (rows + 31) / 32 ? 3 : 2;
}
// ... from which on workgroups of 256 rows take them: 192 rows of 32 x 8000 tokens 327 us, in waves 302; 256: 334, 460 (uniform codes: 144 rows 397, 463; 128: 395, 294).
// Not over few tokens: 256 rows of 2000 31 us, in waves 21.
bool tree_in_blocks(int64_t rows, bool rtn, int64_t tiles) { return rows > (rtn ? 128 : 192) && (tiles >= 4096 || rows > 512); }
template <typename T, int NCW> PagedPlan paged_plan(int64_t batch, int64_t table_pages, int64_t page_tokens, int64_t max_queries, int64_t q_heads, int64_t H, bool tree) {
  PagedPlan p = {};
  const int64_t rows = std::max<int64_t>(max_queries, 1) * (q_heads / H), most = (table_pages * page_tokens + kTile - 1) / kTile;      // tiles of a sequence
  if (sizeof(T) == 2 && tree && tree_in_blocks(rows, is_rtn(NCW), batch * most * H)) {      // one workgroup a CU, pieces of equal size over all sequences
    const int row_blocks = (int)((rows + kTileRows - 1) / kTileRows), room = (int)std::max<int64_t>(256 / (H * row_blocks), 1);
    // Whole sequences, with no results to keep and join, where they are several rounds of workgroups by themselves and none can be much longer than a round: 256 rows of
    // 128 x 4000 tokens 847 us, in pieces 862, of 128 uneven ones 483, 497, one of 4000 among 127 of 500 187, 194; but one of 8000 321, 203, of 16 384 638, 224, of
    // 131 072 4952, 498; of 8000 among 255 358, 365, of 16 384 642, 412.
    const int64_t tokens = table_pages * page_tokens;
    const bool whole = batch >= 4 * room && (tokens <= 4096 || (tokens <= 16384 && batch >= 8 * room));
    const int slots = whole ? 1 : room;
    const int64_t tiles = std::max<int64_t>((table_pages * page_tokens + 63) / 64, 1);
    const int64_t items = slots == 1 ? batch : std::min(batch * tiles, piece_room(slots, (int)batch) + batch);
    if (items * H < (1 << 22)) {                           // (threads of a launch: below 2^32)
      p.row_blocks = row_blocks; p.slots = slots; p.items = items;
      p.results = std::min<int64_t>(items, piece_results(slots, (int)batch));
      p.merge = tiles > 1 && slots > 1;
      p.by_rows = items <= 16 * batch;
      p.many = items > kManyPieces * batch;
      return p;
    }
  }
  if (sizeof(T) == 2 && !tree && rows > kFewRows) {                 // workgroups of 256 rows, one a CU: the tokens in pieces if there are too few of them
    p.row_blocks = (int)((rows + kTileRows - 1) / kTileRows);
    // ... of 4 tiles of 64 at least, of 2 where there is one block of rows and so little to join (180 rows over 700 tokens: 28.0 us, 22.2; 160 over 6000: 34.3, 31.5;
    // 1200 rows over 300: 23.3, 26.2)
    p.slots = (int)std::max<int64_t>(std::min(256 / std::max<int64_t>(batch * H * p.row_blocks, 1), most / (p.row_blocks == 1 ? 4 : 8)), 1);
    p.items = p.results = batch * p.slots;
    p.merge = p.slots > 1;
    p.by_rows = p.slots <= 16;
    p.many = p.slots > kManyPieces;
    return p;
  }
  // 9 to 16 rows fill one column of a wave, but two columns take as long and join their results (16 rows of 8 x 9999 tokens, 3 bits: 37.3 us, in one column
  // 39.7; of one sequence of 12 288: 18.9, 29.8; of 32 x 4000 46.1, 44.8); 8 rows do not (one sequence of 131 072: 49.0, 41.9; 32 x 16 384: 138, 101; 8 x 9999 31.3,
  // 30.4; but one of 16 384 18.0, 19.8).
  p.cols = sizeof(T) == 4 ? 1 : tree ? tree_columns(rows, is_rtn(NCW), batch * most * H) : rows > 8 ? 2 : 1;
  // (threads of a launch: below 2^32, where row tiles share a grid dimension with the pieces)
  if (tree && (batch + 512) * H * ((rows + 31) / 32) >= (1 << 22)) p.cols = 1;
  const int per_wave = 16 * p.cols, waves = p.cols > 1 ? Shape<T, NCW, 2>::kWaves : Shape<T, NCW, 1>::kWaves;
  p.row_tiles = (unsigned)((rows + per_wave - 1) / per_wave);
  // As many pieces as make all waves that the chip holds (32 x 16 384 tokens: 95.7 us, half as many 111, twice as many 99; 5 queries of 8 x 9999 37.7, 42.8,
  // 50.7); the kernel makes fewer of short ones.
  p.slots = (int)std::max<int64_t>((p.cols > 1 ? Shape<T, NCW, 2>::kSlots : Shape<T, NCW, 1>::kSlots) / (H * p.row_tiles), 1);
  if (tree && p.cols > 1) {                                // (whole workgroups of pieces: no more of them than run at once)
    const int64_t at_once = Shape<T, NCW, 2>::kSlots / Shape<T, NCW, 2>::kWaves, groups = std::max<int64_t>(at_once / (H * p.row_tiles), 1);
    p.slots = (int)groups * Shape<T, NCW, 2>::kWaves;
    p.rows_apart = groups % 8 != 0 || batch * most < 4 * p.slots;      // (few tiles a wave: 104 rows over 2000 tokens 16.7 us, on the same CUs 19.6)
  }
  const int64_t pieces = std::min(batch * std::max<int64_t>(most, 1), std::max<int64_t>(p.slots - batch, std::max(p.slots / 2, 1)) + batch);
  if (p.cols > 1) {                                        // (a workgroup has results of as many sequences as it has pieces of)
    const int64_t groups = (pieces + waves - 1) / waves;
    p.blocks = (unsigned)((groups + 7) / 8 * 8 * H);
    if (p.rows_apart) p.blocks = (unsigned)((groups * p.row_tiles + 7) / 8 * 8 * H);
    p.items = p.results = groups + batch;
    p.merge = groups > 1;
  } else {
    p.blocks = (unsigned)((pieces * H + waves - 1) / waves);
    p.items = p.results = pieces;
    p.merge = most > 1;
  }
  p.many = p.items > kManyPieces * batch;
  p.by_rows = p.items <= 8 * batch && batch * max_queries * q_heads >= 512;
  return p;
}

}  // namespace

static PagedPlan plan_of(int dtype, int n_codewords, const PagedAttendArgs& a, bool tree) {
  PagedPlan p = {};
  AQUAKV_PAGED(dtype, n_codewords, (p = paged_plan<T, N>(a.batch, a.table_pages, a.pool.page_tokens, a.max_queries, a.q_heads, a.H, tree)));
  return p;
}

size_t paged_attend_workspace_bytes(int dtype, int n_codewords, const PagedAttendArgs& a, bool tree) {
  const PagedPlan p = plan_of(dtype, n_codewords, a, tree);
  return p.merge ? (size_t)p.results * a.max_queries * a.q_heads * (kGroup + 2) * sizeof(float) + (size_t)a.batch * sizeof(int2) : 0;
}

hipError_t launch_paged_attend(int dtype, int n_codewords, const PagedAttendArgs& args, void* workspace, hipStream_t stream) {
  PagedAttendArgs a = args;
  const PagedPlan plan = plan_of(dtype, n_codewords, a, a.tree != nullptr);
  a.slots = plan.slots;
  a.row_blocks = plan.row_blocks;
  a.items = (int)plan.items;
  a.row_tiles = (int)plan.row_tiles;
  a.rows_apart = (int)plan.rows_apart;
  a.part = static_cast<float*>(workspace);
  a.stats = a.part + plan.results * a.max_queries * a.q_heads * kGroup;
  a.heads = plan.merge ? reinterpret_cast<int2*>(a.stats + plan.results * a.max_queries * a.q_heads * 2) : nullptr;
  a.page_groups = a.pool.page_tokens / 8;
  a.page_magic = a.page_groups == 1 ? 0xffffffffu : (uint32_t)((uint64_t(1) << 32) / a.page_groups);
  if (plan.row_blocks != 0) {
    const hipError_t e = a.tree != nullptr ? launch_paged_tree_tiles(n_codewords, a, stream) : launch_paged_tiles(n_codewords, a, stream);
    if (e) return e;
  } else {
    const dim3 blocks(plan.blocks, plan.rows_apart ? 1u : plan.row_tiles);
    const hipError_t e = a.tree != nullptr ? launch_paged_tree_rows(dtype, n_codewords, plan.cols, blocks, a, stream)
                                           : launch_rows<false>(dtype, n_codewords, plan.cols, blocks, a, stream);
    if (e) return e;
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
