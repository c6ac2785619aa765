// Which tokens of a cache in pages are kept, and the rows of those that are: eviction by accumulated attention weight, and the accepted branch of
// drafted tokens.
#include "codec_core.h"
#include "kernels.h"

namespace aquakv {
namespace {

// Token -> row of the pool (page * page_tokens + place), -1: its page is not in the pool.
struct PageDivider { uint32_t tokens, magic; };
__device__ __forceinline__ int64_t row_of_token(const int32_t* table, int table_pages, const PageDivider& d, int n_pages, int64_t token) {
  if (token < 0 || token >= (int64_t)table_pages * d.tokens) return -1;
  const uint32_t t = (uint32_t)token;
  uint32_t page = (uint32_t)(((uint64_t)t * d.magic) >> 32);                 // (one short at most)
  if (t - page * d.tokens >= d.tokens) ++page;
  const int at = table[page];
  return (uint32_t)at < (uint32_t)n_pages ? (int64_t)at * d.tokens + (t - page * d.tokens) : -1;
}
PageDivider divider(int page_tokens) { return {(uint32_t)page_tokens, (uint32_t)((uint64_t(1) << 32) / (uint32_t)page_tokens)}; }

// ---------------------------------------------------------------- select
// A token's key: larger means kept sooner.  Its mass (heads added up in their order, 32 bits) as an integer of the same order; what is no number comes ahead of
// nothing but a token that is not there.
__device__ __forceinline__ uint32_t key_of(float mass) {
  if (mass != mass) return 1u;
  const uint32_t x = __float_as_uint(mass + 0.0f);         // (-0 is 0)
  return (x >> 31) ? ~x : x | 0x80000000u;
}
constexpr uint32_t kAlways = 0xffffffffu;
__global__ __launch_bounds__(256) void mass_keys_kernel(const PagedSelectArgs a, PageDivider d) {
  const int b = blockIdx.y;
  const int64_t room = (int64_t)a.table_pages * a.page_tokens;
  const int64_t len = min((int64_t)max(a.seq_lens[b], 0), room), t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (t >= len) return;
  const int64_t row = row_of_token(a.page_table + (int64_t)b * a.table_pages, a.table_pages, d, a.n_pages, t);
  uint32_t key = 0u;
  if (row >= 0) {
    if (t < a.n_first || t >= len - a.n_last) {
      key = kAlways;
    } else {
      const int64_t page = row / a.page_tokens;
      const float* const at = a.mass + page * a.H * a.page_tokens + (row - page * a.page_tokens);
      float sum = at[0];
      for (int h = 1; h < a.H; ++h) sum += at[(int64_t)h * a.page_tokens];
      key = key_of(sum);
    }
  }
  a.keys[b * room + t] = key;
}

// One workgroup a sequence: the budget-th largest key by its digits (11, 11, 10 bits), then the tokens above it and the first of those that have it, in order:
// every wave has a run of the tokens and counts its own first.
constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64, kBins = 2048;
__global__ __launch_bounds__(kSelectThreads) void select_kernel(const PagedSelectArgs a) {
  __shared__ uint32_t bins[kBins];
  __shared__ uint32_t sums[kSelectWaves], above[kSelectWaves], equal[kSelectWaves];
  __shared__ uint32_t chosen[2];
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t room = (int64_t)a.table_pages * a.page_tokens;
  const int len = (int)min((int64_t)max(a.seq_lens[b], 0), room), n = min(len, a.budget);
  const uint32_t* const keys = a.keys + b * room;
  int32_t* const kept = a.kept + (int64_t)b * a.budget;
  for (int i = n + tid; i < a.budget; i += kSelectThreads) kept[i] = -1;
  if (tid == 0) a.n_kept[b] = n;
  if (n == 0) return;
  if (len <= a.budget) {
    for (int i = tid; i < n; i += kSelectThreads) kept[i] = i;
    return;
  }
  uint32_t prefix = 0, need = (uint32_t)n;                 // digits found so far; so many are still to be taken among the keys that have them
#pragma unroll 1
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, width = pass == 2 ? 10 : 11, above_shift = shift + width;
    for (int i = tid; i < kBins; i += kSelectThreads) bins[i] = 0;
    __syncthreads();
    for (int i = tid; i < len; i += kSelectThreads) {
      const uint32_t k = keys[i];
      if (pass == 0 || (k >> above_shift) == prefix) atomicAdd(&bins[(k >> shift) & ((1u << width) - 1u)], 1u);
    }
    __syncthreads();
    // sums from the largest digit down: thread i has digits 2047 - 2 i and the one below it
    const uint32_t x = bins[kBins - 1 - 2 * tid], y = bins[kBins - 2 - 2 * tid];
    uint32_t run = x + y;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
      const uint32_t o = __shfl_up(run, s);
      if (lane >= s) run += o;
    }
    if (lane == 63) sums[wave] = run;
    __syncthreads();
    uint32_t before = run - x - y;
    for (int w = 0; w < wave; ++w) before += sums[w];
    if (before < need && before + x >= need) { chosen[0] = kBins - 1 - 2 * tid; chosen[1] = need - before; }
    else if (before + x < need && before + x + y >= need) { chosen[0] = kBins - 2 - 2 * tid; chosen[1] = need - before - x; }
    __syncthreads();
    prefix = prefix << width | chosen[0];
    need = chosen[1];
    __syncthreads();
  }
  // prefix is the last key that is taken, of which the first `need` tokens are
  const int each = ((len + kSelectWaves - 1) / kSelectWaves + 63) & ~63, from = wave * each, to = from + max(min(each, len - from), 0);
  uint32_t more = 0, same = 0;
  for (int i = from + lane; i < to; i += 64) {
    const uint32_t k = keys[i];
    more += k > prefix;
    same += k == prefix;
  }
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    more += __shfl_xor(more, s);
    same += __shfl_xor(same, s);
  }
  if (lane == 0) { above[wave] = more; equal[wave] = same; }
  __syncthreads();
  uint32_t tie = 0, at = 0;                                // of the tokens before this wave's: those that have the last key, those that are kept
  for (int w = 0; w < wave; ++w) { at += above[w]; tie += equal[w]; }
  at += min(tie, need);
  const uint64_t below = (1ull << lane) - 1;
  for (int i0 = from; i0 < to; i0 += 64) {
    const int i = i0 + lane;
    const uint32_t k = i < to ? keys[i] : 0u;
    const uint64_t ties = __builtin_amdgcn_ballot_w64(i < to && k == prefix);
    const bool keep = i < to && (k > prefix || (k == prefix && tie + __builtin_popcountll(ties & below) < need));
    const uint64_t all = __builtin_amdgcn_ballot_w64(keep);
    if (keep) kept[at + __builtin_popcountll(all & below)] = i;
    at += __builtin_popcountll(all);
    tie += __builtin_popcountll(ties);
  }
}

// ---------------------------------------------------------------- keep
// The arrays of a pool as units of 16, 8, 4 or 2 bytes: unit u of a row at row * row_bytes + u * unit, or (mass: [page][head][token]) by page, head and place.
struct KeepArray { uint8_t* p; int units, unit; };
struct KeepLaunch { KeepArray arrays[5]; int n_arrays; PageDivider d; uint8_t* staged; int64_t staged_at[5]; };
__device__ __forceinline__ uint8_t* unit_at(const KeepArray& x, bool mass, const PageDivider& d, int64_t row, int u) {
  if (!mass) return x.p + (row * x.units + u) * x.unit;
  const int64_t page = row / d.tokens;
  return x.p + ((page * x.units + u) * d.tokens + (row - page * d.tokens)) * 4;
}
__device__ __forceinline__ u32x4 load_unit(const uint8_t* p, int unit) {
  u32x4 x = {0, 0, 0, 0};
  if (unit == 16) x = *reinterpret_cast<const u32x4*>(p);
  else if (unit == 8) { const u32x2 y = *reinterpret_cast<const u32x2*>(p); x.x = y.x; x.y = y.y; }
  else if (unit == 4) x.x = *reinterpret_cast<const uint32_t*>(p);
  else x.x = *reinterpret_cast<const uint16_t*>(p);
  return x;
}
__device__ __forceinline__ void store_unit(uint8_t* p, int unit, const u32x4& x) {
  if (unit == 16) *reinterpret_cast<u32x4*>(p) = x;
  else if (unit == 8) *reinterpret_cast<u32x2*>(p) = u32x2{x.x, x.y};
  else if (unit == 4) *reinterpret_cast<uint32_t*>(p) = x.x;
  else *reinterpret_cast<uint16_t*>(p) = (uint16_t)x.x;
}
// Rows that entry i of sequence b goes from and to, -1: nothing to move.
struct Move { int64_t from, to; };
__device__ __forceinline__ Move move_of(const PagedKeepArgs& a, const PageDivider& d, int b, int i) {
  if (i >= min(a.n_kept[b], a.max_kept)) return {-1, -1};
  const int64_t first = a.first != nullptr ? a.first[b] : 0;
  Move m;
  m.from = row_of_token(a.page_table + (int64_t)b * a.table_pages, a.table_pages, d, a.pool.n_pages, a.kept[(int64_t)b * a.max_kept + i]);
  m.to = a.to_table != nullptr ? row_of_token(a.to_table + (int64_t)b * a.to_pages, a.to_pages, d, a.pool.n_pages, first + i)
                               : row_of_token(a.page_table + (int64_t)b * a.table_pages, a.table_pages, d, a.pool.n_pages, first + i);
  if (first < 0 || m.from == m.to) m.from = -1;
  return m;
}

// A workgroup has a column of units of one array and takes it through all entries of a sequence: all reads, then all writes, so that the rows may be
// the same ones in any order.  blockIdx = (array and column, sequence); LANES threads a row.
constexpr int kMoveThreads = 1024, kMoveUnits = 8;
struct Columns { int first[6], lanes; };                   // blockIdx.x from which an array's columns go
template <int UNITS>
__global__ __launch_bounds__(kMoveThreads) void keep_columns_kernel(const PagedKeepArgs a, const KeepLaunch l, const Columns cols) {
  const int b = blockIdx.y;
  int n = 0;
  while (n + 1 < l.n_arrays && (int)blockIdx.x >= cols.first[n + 1]) ++n;
  const bool mass = n == 4;
  const KeepArray x = l.arrays[n];
  const int lanes = mass ? 1 : min(cols.lanes, x.units), column = blockIdx.x - cols.first[n];
  const int per_pass = blockDim.x / lanes, row = threadIdx.x / lanes, u = column * lanes + threadIdx.x % lanes;
  const bool there = row < per_pass && u < x.units;
  u32x4 v[UNITS];
  int64_t to[UNITS];
#pragma unroll
  for (int k = 0; k < UNITS; ++k) {
    const Move m = there ? move_of(a, l.d, b, k * per_pass + row) : Move{-1, -1};
    to[k] = m.from < 0 ? -1 : m.to;
    if (to[k] >= 0) v[k] = load_unit(unit_at(x, mass, l.d, m.from, u), x.unit);
  }
  __builtin_amdgcn_s_waitcnt(0);                           // (every read has come back)
  __syncthreads();
#pragma unroll
  for (int k = 0; k < UNITS; ++k)
    if (to[k] >= 0) store_unit(unit_at(x, mass, l.d, to[k], u), x.unit, v[k]);
}

// A thread takes a unit of an entry's row: from pages to other pages, to the workspace, or back from it.  blockIdx = (block of units, array, sequence).
enum KeepWay : int { kAcross = 0, kOut = 1, kBack = 2 };
template <int WAY>
__global__ __launch_bounds__(256) void keep_rows_kernel(const PagedKeepArgs a, const KeepLaunch l) {
  const int b = blockIdx.z, n = blockIdx.y;
  const bool mass = n == 4;
  const KeepArray x = l.arrays[n];
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int i = (int)(mass ? id % a.max_kept : id / x.units), u = (int)(mass ? id / a.max_kept : id - (int64_t)i * x.units);
  if (i >= a.max_kept || u >= x.units) return;
  const Move m = move_of(a, l.d, b, i);
  if (m.from < 0 || m.to < 0) return;
  uint8_t* const staged = l.staged + l.staged_at[n] + ((int64_t)b * a.max_kept * x.units + id) * x.unit;
  const uint8_t* const from = WAY == kBack ? staged : unit_at(x, mass, l.d, m.from, u);
  uint8_t* const to = WAY == kOut ? staged : unit_at(x, mass, l.d, m.to, u);
  store_unit(to, x.unit, load_unit(from, x.unit));
}

int unit_of(int64_t bytes) { return bytes % 16 == 0 ? 16 : bytes % 8 == 0 ? 8 : bytes % 4 == 0 ? 4 : 2; }
KeepLaunch keep_launch(const PagedKeepArgs& a) {
  KeepLaunch l = {};
  const int64_t bytes[4] = {a.code_row, a.scale_row, a.code_row, a.scale_row};
  uint8_t* const p[4] = {a.pool.k_codes, reinterpret_cast<uint8_t*>(a.pool.k_scales), a.pool.v_codes, reinterpret_cast<uint8_t*>(a.pool.v_scales)};
  for (int i = 0; i < 4; ++i) l.arrays[i] = {p[i], (int)(bytes[i] / unit_of(bytes[i])), unit_of(bytes[i])};
  l.arrays[4] = {reinterpret_cast<uint8_t*>(a.mass), a.H, 4};
  l.n_arrays = a.mass != nullptr ? 5 : 4;
  l.d = divider(a.pool.page_tokens);
  return l;
}
// Rows in place whose column a workgroup can hold.
constexpr int kMostHeld = kMoveThreads * kMoveUnits;

}  // namespace

size_t paged_select_workspace_bytes(int64_t batch, int64_t table_pages, int64_t page_tokens) { return (size_t)(batch * table_pages * page_tokens) * sizeof(uint32_t); }

hipError_t launch_paged_select(const PagedSelectArgs& a, hipStream_t stream) {
  const int64_t room = (int64_t)a.table_pages * a.page_tokens;
  mass_keys_kernel<<<dim3((unsigned)((room + 255) / 256), (unsigned)a.batch), 256, 0, stream>>>(a, divider(a.page_tokens));
  if (const hipError_t e = hipGetLastError()) return e;
  select_kernel<<<(unsigned)a.batch, kSelectThreads, 0, stream>>>(a);
  return hipGetLastError();
}

size_t paged_keep_workspace_bytes(int64_t batch, int64_t max_kept, int64_t code_row, int64_t scale_row, int64_t H, bool mass) {
  if (max_kept <= kMostHeld) return 0;
  size_t n = 0;
  const int64_t bytes[5] = {code_row, scale_row, code_row, scale_row, mass ? 4 * H : 0};
  for (const int64_t x : bytes) n += ((size_t)(batch * max_kept * x) + 255) & ~(size_t)255;
  return n;
}

hipError_t launch_paged_keep(const PagedKeepArgs& a, void* workspace, hipStream_t stream) {
  KeepLaunch l = keep_launch(a);
  if (a.to_table == nullptr && a.max_kept <= kMostHeld) {
    Columns cols = {};
    cols.lanes = std::min(8, kMostHeld / a.max_kept);
    cols.lanes = cols.lanes >= 8 ? 8 : cols.lanes >= 4 ? 4 : cols.lanes >= 2 ? 2 : 1;
    int most = 1, at = 0;
    for (int i = 0; i < l.n_arrays; ++i) {
      const int lanes = i == 4 ? 1 : std::min(cols.lanes, l.arrays[i].units);
      cols.first[i] = at;
      at += (l.arrays[i].units + lanes - 1) / lanes;
      most = std::max(most, lanes);
    }
    cols.first[l.n_arrays] = at;
    // threads for all entries at once, up to a workgroup's; what is more goes into registers
    const int threads = std::min<int64_t>(((int64_t)a.max_kept * most + 63) / 64 * 64, kMoveThreads);
    const int units = (a.max_kept + threads / most - 1) / (threads / most);
    const dim3 grid((unsigned)at, (unsigned)a.batch);
    if (units <= 1) keep_columns_kernel<1><<<grid, threads, 0, stream>>>(a, l, cols);
    else if (units <= 2) keep_columns_kernel<2><<<grid, threads, 0, stream>>>(a, l, cols);
    else if (units <= 4) keep_columns_kernel<4><<<grid, threads, 0, stream>>>(a, l, cols);
    else keep_columns_kernel<8><<<grid, threads, 0, stream>>>(a, l, cols);
    return hipGetLastError();
  }
  int64_t most = 0, at = 0;
  l.staged = static_cast<uint8_t*>(workspace);
  for (int i = 0; i < l.n_arrays; ++i) {
    most = std::max<int64_t>(most, (int64_t)a.max_kept * l.arrays[i].units);
    l.staged_at[i] = at;
    at += ((int64_t)a.batch * a.max_kept * l.arrays[i].units * l.arrays[i].unit + 255) & ~(int64_t)255;
  }
  const dim3 grid((unsigned)((most + 255) / 256), (unsigned)l.n_arrays, (unsigned)a.batch);
  if (a.to_table != nullptr) {
    keep_rows_kernel<kAcross><<<grid, 256, 0, stream>>>(a, l);
    return hipGetLastError();
  }
  keep_rows_kernel<kOut><<<grid, 256, 0, stream>>>(a, l);
  if (const hipError_t e = hipGetLastError()) return e;
  keep_rows_kernel<kBack><<<grid, 256, 0, stream>>>(a, l);
  return hipGetLastError();
}

}  // namespace aquakv
