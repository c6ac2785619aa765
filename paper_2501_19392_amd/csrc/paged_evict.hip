// Which tokens of a cache in pages are kept, and the rows of those that are: eviction by accumulated attention weight, and the accepted branch of
// drafted tokens.
#include "codec_core.h"
#include "kernels.h"

namespace aquakv {
namespace {

struct PageDivider { uint32_t tokens, magic; };
struct InPage { uint32_t page, in; };                      // token / tokens of a page, and the rest
__device__ __forceinline__ InPage in_page(const PageDivider& d, uint32_t token) {
  uint32_t page = (uint32_t)(((uint64_t)token * d.magic) >> 32);             // (one short at most)
  if (token - page * d.tokens >= d.tokens) ++page;
  return {page, token - page * d.tokens};
}
// Token -> its page in the pool, -1: not there; its place in the page.
struct Place { int page; uint32_t in; };
__device__ __forceinline__ Place place_of_token(const int32_t* table, int table_pages, const PageDivider& d, int n_pages, int64_t token) {
  if (token < 0 || token >= (int64_t)table_pages * d.tokens) return {-1, 0u};
  const InPage t = in_page(d, (uint32_t)token);
  const int at = table[t.page];
  return {(uint32_t)at < (uint32_t)n_pages ? at : -1, t.in};
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
__device__ __forceinline__ int cached(const PagedSelectArgs& a, int b) { return (int)min((int64_t)max(a.seq_lens[b], 0), (int64_t)a.table_pages * a.page_tokens); }
// The keys of N tokens, `step` apart from t on, for those below `to` (at least one token; the others: anything).  Without branches, so that the tokens' pages are
// looked up together, then their masses, kHeads of each at once: one sequence of 131 072 tokens to 32 768 45.9 us with the moves, one token after the other 47.3.
template <int N> __device__ __forceinline__ void token_keys(const PagedSelectArgs& a, const PageDivider& d, int b, int len, int t, int step, int to, uint32_t (&key)[N]) {
  constexpr int kHeads = 4;
  const int32_t* const table = a.page_table + (int64_t)b * a.table_pages;
  uint32_t in[N];
  int page[N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const uint32_t token = (uint32_t)min((int64_t)t + (int64_t)k * step, (int64_t)to - 1);
    const InPage p = in_page(d, token);
    in[k] = p.in;
    page[k] = table[p.page];
    key[k] = (int)token < a.n_first || (int)token >= len - a.n_last ? kAlways : 1u;
  }
  const float* at[N];
  float sum[N] = {};
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const bool there = (uint32_t)page[k] < (uint32_t)a.n_pages;
    at[k] = a.mass + (int64_t)(there ? page[k] : 0) * a.H * a.page_tokens + in[k];
    if (!there) key[k] = 0u;
  }
  for (int h = 0; h < a.H; h += kHeads) {                  // (added in order)
    float x[N][kHeads];
#pragma unroll
    for (int i = 0; i < kHeads; ++i)
#pragma unroll
      for (int k = 0; k < N; ++k) x[k][i] = at[k][(int64_t)min(h + i, a.H - 1) * a.page_tokens];
#pragma unroll
    for (int i = 0; i < kHeads; ++i)
#pragma unroll
      for (int k = 0; k < N; ++k) sum[k] = h + i < a.H ? sum[k] + x[k][i] : sum[k];
  }
#pragma unroll
  for (int k = 0; k < N; ++k)
    if (key[k] == 1u) key[k] = key_of(sum[k]);
}

// The budget-th largest key digit by digit: 11, 11 and 10 bits.  What is known of it ahead of a digit: the ones before it, and how many tokens are still to be taken
// among the keys that have those.
constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64, kBins = 2048;
__device__ __forceinline__ int shift_of(int digit) { return digit == 0 ? 21 : digit == 1 ? 10 : 0; }
__device__ __forceinline__ int width_of(int digit) { return digit == 2 ? 10 : 11; }
struct Known { uint32_t prefix, need; };
struct Scan { uint32_t sums[kSelectWaves], chosen[2]; };
// Thread i has the counts of digits 2047 - 2 i (x) and the one below it (y).
__device__ __forceinline__ Known next_digit(Known k, int digit, uint32_t x, uint32_t y, Scan& s) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t run = x + y;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t o = __shfl_up(run, d);
    if (lane >= d) run += o;
  }
  if (lane == 63) s.sums[wave] = run;
  __syncthreads();
  uint32_t before = run - x - y;
  for (int w = 0; w < wave; ++w) before += s.sums[w];
  if (before < k.need && before + x >= k.need) { s.chosen[0] = kBins - 1 - 2 * tid; s.chosen[1] = k.need - before; }
  else if (before + x < k.need && before + x + y >= k.need) { s.chosen[0] = kBins - 2 - 2 * tid; s.chosen[1] = k.need - before - x; }
  __syncthreads();
  k = {k.prefix << width_of(digit) | s.chosen[0], s.chosen[1]};
  __syncthreads();
  return k;
}
// Whether a key counts for a digit, and for which value of it.
__device__ __forceinline__ bool counts(uint32_t key, const Known& k, int digit) { return digit == 0 || key >> (shift_of(digit) + width_of(digit)) == k.prefix; }
__device__ __forceinline__ uint32_t digit_of(uint32_t key, int digit) { return (key >> shift_of(digit)) & ((1u << width_of(digit)) - 1u); }
// The tokens of a run that are kept, in order: `at` of this sequence's, and `tie` that have the last key, lie before it.  64 at a time, one wave.
template <typename Key> __device__ __forceinline__ void emit(int32_t* kept, const Known& k, uint32_t at, uint32_t tie, int from, int to, const Key& key) {
  const int lane = threadIdx.x & 63;
  const uint64_t below = (1ull << lane) - 1;
  for (int i0 = from; i0 < to; i0 += 64) {
    const int i = i0 + lane;
    const uint32_t x = i < to ? key(i) : 0u;
    const uint64_t ties = __builtin_amdgcn_ballot_w64(i < to && x == k.prefix);
    const bool keep = i < to && (x > k.prefix || (x == k.prefix && tie + __builtin_popcountll(ties & below) < k.need));
    const uint64_t all = __builtin_amdgcn_ballot_w64(keep);
    if (keep) kept[at + __builtin_popcountll(all & below)] = i;
    at += __builtin_popcountll(all);
    tie += __builtin_popcountll(ties);
  }
}
__device__ __forceinline__ uint32_t wave_sum(uint32_t x) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d);
  return x;
}
// Everything but the choice: what is behind the tokens that are kept, and sequences that keep all of theirs.  -> whether that was all
// (counted without a sign: a step past a budget or length near 2^31 stays above it)
__device__ __forceinline__ bool keeps_all(const PagedSelectArgs& a, int b, int len, int tid, int threads) {
  const int n = min(len, a.budget);
  int32_t* const kept = a.kept + (int64_t)b * a.budget;
  for (uint32_t i = n + tid; i < (uint32_t)a.budget; i += threads) kept[i] = -1;
  if (tid == 0) a.n_kept[b] = n;
  if (n != 0 && len <= a.budget)
    for (uint32_t i = tid; i < (uint32_t)n; i += threads) kept[i] = (int32_t)i;
  return n == 0 || len <= a.budget;
}

// One workgroup a sequence, keys in LDS: 12.4 us for 32 sequences of up to 4160 tokens of 8 heads (4 MB of mass), a chain of some twenty barriers: nothing in it is large.
constexpr int kHeldKeys = 16384;
template <int KEYS> __global__ __launch_bounds__(kSelectThreads) void select_held_kernel(const PagedSelectArgs a, const PageDivider d) {
  __shared__ uint32_t keys[KEYS];
  __shared__ uint32_t bins[kBins];
  __shared__ uint32_t above[kSelectWaves], equal[kSelectWaves];
  __shared__ Scan scan;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, len = cached(a, b);
  if (keeps_all(a, b, len, tid, kSelectThreads)) return;
  for (int i = tid; i < kBins; i += kSelectThreads) bins[i] = 0;
  __syncthreads();
  constexpr int kAtOnce = 8;
  for (int i0 = 0; i0 < len; i0 += kAtOnce * kSelectThreads) {
    uint32_t x[kAtOnce];
    token_keys(a, d, b, len, i0 + tid, kSelectThreads, len, x);
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int i = i0 + k * kSelectThreads + tid;
      if (i >= len) break;
      keys[i] = x[k];
      atomicAdd(&bins[digit_of(x[k], 0)], 1u);                               // (adding up those of a wave first takes longer: 16.8 us)
    }
  }
  __syncthreads();
  Known k = {0u, (uint32_t)a.budget};
  for (int digit = 0;;) {
    k = next_digit(k, digit, bins[kBins - 1 - 2 * tid], bins[kBins - 2 - 2 * tid], scan);
    if (++digit == 3) break;
    for (int i = tid; i < kBins; i += kSelectThreads) bins[i] = 0;
    __syncthreads();
    for (int i = tid; i < len; i += kSelectThreads)
      if (counts(keys[i], k, digit)) atomicAdd(&bins[digit_of(keys[i], digit)], 1u);
    __syncthreads();
  }
  // a run of the tokens for each wave, which counts what it keeps first
  const int each = ((len + kSelectWaves - 1) / kSelectWaves + 63) & ~63, from = min(wave * each, len), to = from + min(each, len - from);
  uint32_t more = 0, same = 0;
  for (int i = from + lane; i < to; i += 64) {
    more += keys[i] > k.prefix;
    same += keys[i] == k.prefix;
  }
  more = wave_sum(more);
  same = wave_sum(same);
  if (lane == 0) { above[wave] = more; equal[wave] = same; }
  __syncthreads();
  uint32_t at = 0, tie = 0;
  for (int w = 0; w < wave; ++w) { at += above[w]; tie += equal[w]; }
  emit(a.kept + (int64_t)b * a.budget, k, at + min(tie, k.need), tie, from, to, [&](int i) { return keys[i]; });
}

// Long sequences: a workgroup a slab of at least kSlab tokens, of which there are at most kMostSlabs, a launch a digit.  Each counts its slab's keys by the digit; the
// next launch adds the slabs up (every workgroup for itself) and counts the digit behind it; the last one writes the tokens.  131 072 tokens: 5.4, 7.8, 7.6 and 10.2 us, of which
// a launch that reads 256 KB of counts from the caches is most (one workgroup for all of it: 140 us).
constexpr int kSlab = 4096, kMostSlabs = 256, kHeld = kSlab / kSelectThreads;
struct Slabs {
  uint32_t* counts;                                        // [batch, 3, n, kBins]
  uint32_t* above;                                         // [batch, 2, n]: keys of a slab above the last one by their first, second digit
  Known* known;                                            // [batch, 2]: behind the first, second digit
  int n, tokens;                                           // slabs that there is room for; tokens of each, a multiple of kSlab
};
__device__ __forceinline__ int slabs_of(const Slabs& s, int len) { return (int)(((int64_t)len + s.tokens - 1) / s.tokens); }
// The next digit, and of the counts that it goes by: keys above it and at it, of slab `slab` (own) or of all before it.  (The thread's share: to be added up.)
struct Found { Known k; uint32_t above, at; };
__device__ __forceinline__ Found found(const Slabs& s, Known k, int b, int digit, int slabs, int slab, bool own, Scan& scan) {
  uint32_t x = 0, y = 0, px = 0, py = 0;
  const uint32_t* const from = s.counts + ((int64_t)b * 3 + digit) * s.n * kBins + kBins - 2 - 2 * threadIdx.x;
#pragma unroll 16
  for (int i = 0; i < slabs; ++i) {
    const u32x2 c = *reinterpret_cast<const u32x2*>(from + (int64_t)i * kBins);
    x += c.y;
    y += c.x;
    if (own ? i == slab : i < slab) { px += c.y; py += c.x; }
  }
  Found f;
  f.k = next_digit(k, digit, x, y, scan);
  const uint32_t last = digit_of(f.k.prefix << shift_of(digit), digit), bx = kBins - 1 - 2 * threadIdx.x, by = bx - 1;
  f.above = (bx > last ? px : 0u) + (by > last ? py : 0u);
  f.at = (bx == last ? px : 0u) + (by == last ? py : 0u);
  return f;
}
template <int DIGIT> __global__ __launch_bounds__(kSelectThreads) void slab_counts_kernel(const PagedSelectArgs a, const PageDivider d, const Slabs s) {
  __shared__ uint32_t bins[kBins];
  __shared__ uint32_t above;
  __shared__ Scan scan;
  const int b = blockIdx.y, slab = blockIdx.x, tid = threadIdx.x, len = cached(a, b), slabs = slabs_of(s, len);
  if (slab >= slabs || len <= a.budget || a.budget == 0) return;
  for (int i = tid; i < kBins; i += kSelectThreads) bins[i] = 0;
  if (tid == 0) above = 0;
  Known k = {0u, (uint32_t)a.budget};
  uint32_t* const keys = a.keys + (int64_t)b * s.n * s.tokens;
  const int from = slab * s.tokens, to = from + min(s.tokens, len - from);
  uint32_t held[kHeld];                                    // the first ones, on their way while the digit before is found
  if constexpr (DIGIT > 0) {
#pragma unroll
    for (int i = 0; i < kHeld; ++i) held[i] = keys[min(from + i * kSelectThreads + tid, to - 1)];
    if (DIGIT == 2) k = s.known[2 * b];
    const Found f = found(s, k, b, DIGIT - 1, slabs, slab, true, scan);
    k = f.k;
    const uint32_t more = wave_sum(f.above);
    if ((tid & 63) == 0) atomicAdd(&above, more);
    if (slab == 0 && tid == 0) s.known[2 * b + DIGIT - 1] = k;
  }
  __syncthreads();
  if (DIGIT > 0 && tid == 0) s.above[((int64_t)b * 2 + DIGIT - 1) * s.n + slab] = above;
  if constexpr (DIGIT == 0) {
    for (int t = from; t < to; t += kHeld * kSelectThreads) {
      token_keys(a, d, b, len, t + tid, kSelectThreads, to, held);
#pragma unroll
      for (int i = 0; i < kHeld; ++i) {
        if (t + tid >= to - i * kSelectThreads) break;
        keys[t + tid + i * kSelectThreads] = held[i];
        atomicAdd(&bins[digit_of(held[i], 0)], 1u);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
      if (from + i * kSelectThreads + tid < to && counts(held[i], k, DIGIT)) atomicAdd(&bins[digit_of(held[i], DIGIT)], 1u);
#pragma unroll 4
    for (int t = from + kHeld * kSelectThreads + tid; t < to; t += kSelectThreads) {
      const uint32_t x = keys[t];
      if (counts(x, k, DIGIT)) atomicAdd(&bins[digit_of(x, DIGIT)], 1u);
    }
  }
  __syncthreads();
  uint32_t* const out = s.counts + (((int64_t)b * 3 + DIGIT) * s.n + slab) * kBins;
  for (int i = tid; i < kBins; i += kSelectThreads) out[i] = bins[i];
}
__global__ __launch_bounds__(kSelectThreads) void slab_emit_kernel(const PagedSelectArgs a, const Slabs s) {
  __shared__ Scan scan;
  __shared__ uint32_t above[kSelectWaves], equal[kSelectWaves], before[2];
  const int b = blockIdx.y, slab = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, len = cached(a, b), slabs = slabs_of(s, len);
  if (len <= a.budget || a.budget == 0) {
    keeps_all(a, b, len, slab * kSelectThreads + tid, s.n * kSelectThreads);
    return;
  }
  if (slab >= slabs) return;
  if (slab == 0 && tid == 0) a.n_kept[b] = a.budget;
  if (tid < 2) before[tid] = 0;
  const uint32_t* const keys = a.keys + (int64_t)b * s.n * s.tokens;
  const int each = s.tokens / kSelectWaves, from = (int)min((int64_t)slab * s.tokens + wave * each, (int64_t)len), to = from + min(each, len - from);
  uint32_t held[kHeld];                                    // the first ones, on their way while the last digit is found
#pragma unroll
  for (int i = 0; i < kHeld; ++i) held[i] = keys[min(from + 64 * i + lane, len - 1)];
  const Found f = found(s, s.known[2 * b + 1], b, 2, slabs, slab, false, scan);
  const Known k = f.k;
  __syncthreads();
  // of the slabs before this one: keys above the last one, and those that have it
  uint32_t more = f.above, same = f.at;
  for (int i = tid; i < 2 * slab; i += kSelectThreads) more += s.above[((int64_t)b * 2 + (i >= slab)) * s.n + (i >= slab ? i - slab : i)];
  more = wave_sum(more);
  same = wave_sum(same);
  if (lane == 0) {
    atomicAdd(&before[0], more);
    atomicAdd(&before[1], same);
  }
  more = same = 0;
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    more += from + 64 * i + lane < to && held[i] > k.prefix;
    same += from + 64 * i + lane < to && held[i] == k.prefix;
  }
  for (int i = from + 64 * kHeld + lane; i < to; i += 64) {
    const uint32_t x = keys[i];
    more += x > k.prefix;
    same += x == k.prefix;
  }
  more = wave_sum(more);
  same = wave_sum(same);
  if (lane == 0) { above[wave] = more; equal[wave] = same; }
  __syncthreads();
  uint32_t at = before[0], tie = before[1];
  for (int w = 0; w < wave; ++w) { at += above[w]; tie += equal[w]; }
  emit(a.kept + (int64_t)b * a.budget, k, at + min(tie, k.need), tie, from, to, [&](int i) { return keys[i]; });
}

// ---------------------------------------------------------------- keep
// The arrays of a pool as units of 16, 8, 4 or 2 bytes: a row's lie side by side, those of mass ([page][head][token]) page_tokens apart.
struct KeepArray { uint8_t* p; int units, unit; };
struct KeepLaunch { KeepArray arrays[5]; int n_arrays, row_lanes; PageDivider d; uint8_t* staged; int64_t staged_at[5]; };
__device__ __forceinline__ uint8_t* unit_at(const KeepArray& x, bool mass, const PageDivider& d, const Place& at, int u) {
  if (!mass) return x.p + (((int64_t)at.page * d.tokens + at.in) * x.units + u) * x.unit;
  return x.p + (((int64_t)at.page * x.units + u) * d.tokens + at.in) * 4;
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
  if (unit == 16) __builtin_nontemporal_store(x, reinterpret_cast<u32x4*>(p));
  else if (unit == 8) *reinterpret_cast<u32x2*>(p) = u32x2{x.x, x.y};
  else if (unit == 4) *reinterpret_cast<uint32_t*>(p) = x.x;
  else *reinterpret_cast<uint16_t*>(p) = (uint16_t)x.x;
}
__device__ __forceinline__ Place place_of_row(const PageDivider& d, int row) {
  const InPage r = in_page(d, (uint32_t)row);
  return {(int)r.page, r.in};
}
// Places that entry i of sequence b goes from and to, page -1: nothing to move.
struct Move { Place from, to; };
__device__ __forceinline__ Move move_of(const PagedKeepArgs& a, const PageDivider& d, int b, int i) {
  const Place none = {-1, 0u};
  if (i >= min(a.n_kept[b], a.max_kept)) return {none, none};
  const int64_t first = a.first != nullptr ? a.first[b] : 0;
  const int32_t* const table = a.page_table + (int64_t)b * a.table_pages;
  const Place from = place_of_token(table, a.table_pages, d, a.pool.n_pages, a.kept[(int64_t)b * a.max_kept + i]);
  const Place to = a.to_table != nullptr ? place_of_token(a.to_table + (int64_t)b * a.to_pages, a.to_pages, d, a.pool.n_pages, first + i)
                                         : place_of_token(table, a.table_pages, d, a.pool.n_pages, first + i);
  if (first < 0 || from.page < 0 || to.page < 0 || (from.page == to.page && from.in == to.in)) return {none, none};
  return {from, to};
}

// In place: a workgroup takes a column of up to 128 bytes of one array's rows through the entries of a sequence, a round of them after the other.  As entries ascend, none
// of the rows that a round writes is read later, so that two rounds more are on their way meanwhile; within a round all reads come back before anything is
// written.  32 x 3800 of 4000 rows 69 us, 3.7 TB/s (a copy 5.2); what is left are the rounds' waits, for few sequences all there is.  blockIdx = (array and column,
// sequence).
constexpr int kMoveThreads = 1024, kMoveUnits = 2, kMoveLanes = 8, kMoveChunk = 4096;
struct Columns { int first[6]; };                          // blockIdx.x from which an array's columns go
template <int UNITS, int CHUNK>
__global__ __launch_bounds__(kMoveThreads) void keep_in_place_kernel(const PagedKeepArgs a, const KeepLaunch l, const Columns cols) {
  __shared__ int2 rows[CHUNK];                             // that a chunk's entries go from and to, -1: nothing to move
  const int b = blockIdx.y;
  int n = 0;
  while (n + 1 < l.n_arrays && (int)blockIdx.x >= cols.first[n + 1]) ++n;
  const bool mass = n == 4;
  const KeepArray x = l.arrays[n];
  const int lanes = mass ? 1 : min(kMoveLanes, x.units), column = blockIdx.x - cols.first[n];
  const int per_pass = blockDim.x / lanes, row = threadIdx.x / lanes, u = column * lanes + threadIdx.x % lanes, round = per_pass * UNITS;
  const bool there = row < per_pass && u < x.units;
  const int count = min(a.n_kept[b], a.max_kept);
  const auto at = [&](int row) { return mass ? unit_at(x, true, l.d, place_of_row(l.d, row), u) : x.p + ((int64_t)row * x.units + u) * x.unit; };
  struct Set { u32x4 v[UNITS]; };
  for (int c0 = 0; c0 < count; c0 += CHUNK) {
    const int entries = min(CHUNK, count - c0);
    __syncthreads();
    for (int i = threadIdx.x; i < entries; i += blockDim.x) {
      const Move m = move_of(a, l.d, b, c0 + i);
      rows[i] = m.from.page < 0 ? int2{-1, -1} : int2{(int)(m.from.page * l.d.tokens + m.from.in), (int)(m.to.page * l.d.tokens + m.to.in)};
    }
    __syncthreads();
    const auto request = [&](Set& set, int i0) {
#pragma unroll
      for (int k = 0; k < UNITS; ++k) {
        const int i = i0 + k * per_pass + row;
        const int from = there && i < entries ? rows[i].x : -1;
        if (from >= 0) set.v[k] = load_unit(at(from), x.unit);
      }
    };
    const auto finish = [&](Set& set, int i0, Set& next) { // a round is written, the one two behind it requested
#pragma unroll
      for (int k = 0; k < UNITS; ++k) asm volatile("" : "+v"(set.v[k].x), "+v"(set.v[k].y), "+v"(set.v[k].z), "+v"(set.v[k].w));      // (its reads have come back)
      __syncthreads();
      request(next, i0 + 2 * round);
#pragma unroll
      for (int k = 0; k < UNITS; ++k) {
        const int i = i0 + k * per_pass + row;
        const int to = there && i < entries ? rows[i].y : -1;
        if (to >= 0) store_unit(at(to), x.unit, set.v[k]);
      }
    };
    Set s0 = {}, s1 = {}, s2 = {};
    request(s0, 0);
    request(s1, round);
    for (int i0 = 0; i0 < entries; i0 += 3 * round) {
      finish(s0, i0, s2);
      finish(s1, i0 + round, s0);
      finish(s2, i0 + 2 * round, s1);
    }
  }
}

// kRowsEach entries a workgroup, whose places are worked out first: from pages to other pages, to the workspace, or back from it.  Bound by memory: 94 000 rows of 1 KB to other
// pages 48 us, 4.3 TB/s; stores that went by the L2s' lines took 60 (as they are what is written and not read again).  blockIdx = (entries, sequence).
enum KeepWay : int { kAcross = 0, kOut = 1, kBack = 2 };
constexpr int kRowsEach = 32, kAhead = 8;
template <int WAY> __global__ __launch_bounds__(256) void keep_rows_kernel(const PagedKeepArgs a, const KeepLaunch l) {
  __shared__ Move moves[kRowsEach];
  const int b = blockIdx.y, e0 = blockIdx.x * kRowsEach, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  if (threadIdx.x < kRowsEach) moves[threadIdx.x] = move_of(a, l.d, b, e0 + threadIdx.x);
  __syncthreads();
  const auto staged = [&](int n, int e, int u) { return l.staged + l.staged_at[n] + (((int64_t)b * a.max_kept + e0 + e) * l.arrays[n].units + u) * l.arrays[n].unit; };
  // codes, units of 16 bytes: l.row_lanes lanes a row (keys, then values), kAhead rows of each in flight
  const int rows = 64 / l.row_lanes, each = l.arrays[0].units;
  for (int u = lane & (l.row_lanes - 1); u < 2 * each; u += l.row_lanes) {
    const bool values = u >= each;
    const KeepArray x = {values ? l.arrays[2].p : l.arrays[0].p, each, 16};
    const int at = values ? u - each : u, n = values ? 2 : 0;
    for (int base = wave * rows + lane / l.row_lanes; base < kRowsEach; base += 4 * rows * kAhead) {
      u32x4 v[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int e = base + 4 * rows * k;
        if (e < kRowsEach && moves[e].from.page >= 0) v[k] = *reinterpret_cast<const u32x4*>(WAY == kBack ? staged(n, e, at) : unit_at(x, false, l.d, moves[e].from, at));
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int e = base + 4 * rows * k;
        if (e < kRowsEach && moves[e].from.page >= 0) {
          if (WAY == kOut) *reinterpret_cast<u32x4*>(staged(n, e, at)) = v[k];
          else store_unit(unit_at(x, false, l.d, moves[e].to, at), 16, v[k]);
        }
      }
    }
  }
  for (int n = 1; n < l.n_arrays; n += n == 3 ? 1 : 2) {   // scales, mass
    const bool mass = n == 4;
    const KeepArray x = l.arrays[n];
    for (int i = threadIdx.x; i < kRowsEach * x.units; i += 256) {
      const int e = i % kRowsEach, u = i / kRowsEach;
      if (moves[e].from.page < 0) continue;
      store_unit(WAY == kOut ? staged(n, e, u) : unit_at(x, mass, l.d, moves[e].to, u), x.unit,
                 load_unit(WAY == kBack ? staged(n, e, u) : unit_at(x, mass, l.d, moves[e].from, u), x.unit));
    }
  }
}

int unit_of(int64_t bytes) { return bytes % 16 == 0 ? 16 : bytes % 8 == 0 ? 8 : bytes % 4 == 0 ? 4 : 2; }
KeepLaunch keep_launch(const PagedKeepArgs& a) {
  KeepLaunch l = {};
  const int64_t bytes[4] = {a.code_row, a.scale_row, a.code_row, a.scale_row};
  uint8_t* const p[4] = {a.pool.k_codes, reinterpret_cast<uint8_t*>(a.pool.k_scales), a.pool.v_codes, reinterpret_cast<uint8_t*>(a.pool.v_scales)};
  for (int i = 0; i < 4; ++i) l.arrays[i] = {p[i], (int)(bytes[i] / unit_of(bytes[i])), unit_of(bytes[i])};
  l.arrays[4] = {reinterpret_cast<uint8_t*>(a.mass), a.H, 4};
  l.n_arrays = a.mass != nullptr ? 5 : 4;
  for (l.row_lanes = 1; l.row_lanes < 64 && l.row_lanes < 2 * l.arrays[0].units; l.row_lanes *= 2) {}
  l.d = divider(a.pool.page_tokens);
  return l;
}
// In place through the workspace, in two launches: few sequences of many entries, whose columns are too few workgroups (1 x 3800 entries: 17.3 us, by columns 23.6; 1 x 20 000:
// 28.4, 134; 8 x 7900, 64 columns: 61, 58; 32 x 3800: 104, 69; 1 x 900: 16.4, 9.5).
bool through_workspace(int64_t batch, int64_t max_kept, int64_t code_row) { return max_kept > 1024 && batch * 2 * ((code_row + 127) / 128) < 64; }

}  // namespace

namespace {
// One workgroup a sequence for short ones, otherwise slabs (1 x 12 000 tokens 24.0 us with the moves, in slabs 29.2; 1 x 24 000 36.5, 32.1; 16 x 16 000 42.1, 42.0).
bool keys_held(int64_t room) { return room <= kHeldKeys; }
int64_t slab_tokens(int64_t room) { return ((room + kMostSlabs - 1) / kMostSlabs + kSlab - 1) / kSlab * kSlab; }
int64_t slabs_of(int64_t room) { return (room + slab_tokens(room) - 1) / slab_tokens(room); }
}  // namespace

size_t paged_select_workspace_bytes(int64_t batch, int64_t table_pages, int64_t page_tokens) {
  const int64_t room = table_pages * page_tokens;
  return keys_held(room) ? 0 : (size_t)(batch * slabs_of(room)) * (slab_tokens(room) + 3 * kBins + 2) * sizeof(uint32_t) + (size_t)batch * 2 * sizeof(Known);
}

hipError_t launch_paged_select(const PagedSelectArgs& a, void* workspace, hipStream_t stream) {
  PagedSelectArgs args = a;
  const int64_t room = (int64_t)a.table_pages * a.page_tokens;
  const PageDivider d = divider(a.page_tokens);
  if (keys_held(room)) {
    if (room <= 8192) select_held_kernel<8192><<<(unsigned)a.batch, kSelectThreads, 0, stream>>>(args, d);
    else select_held_kernel<kHeldKeys><<<(unsigned)a.batch, kSelectThreads, 0, stream>>>(args, d);
    return hipGetLastError();
  }
  const int64_t n = slabs_of(room);
  args.keys = static_cast<uint32_t*>(workspace);
  Slabs s = {};
  s.n = (int)n;
  s.tokens = (int)slab_tokens(room);
  s.counts = args.keys + a.batch * n * s.tokens;
  s.known = reinterpret_cast<Known*>(s.counts + a.batch * 3 * n * kBins);
  s.above = reinterpret_cast<uint32_t*>(s.known + 2 * a.batch);
  const dim3 grid((unsigned)n, (unsigned)a.batch);
  slab_counts_kernel<0><<<grid, kSelectThreads, 0, stream>>>(args, d, s);
  slab_counts_kernel<1><<<grid, kSelectThreads, 0, stream>>>(args, d, s);
  slab_counts_kernel<2><<<grid, kSelectThreads, 0, stream>>>(args, d, s);
  slab_emit_kernel<<<grid, kSelectThreads, 0, stream>>>(args, s);
  return hipGetLastError();
}

size_t paged_keep_workspace_bytes(int64_t batch, int64_t max_kept, int64_t code_row, int64_t scale_row, int64_t H, bool mass) {
  if (!through_workspace(batch, max_kept, code_row)) return 0;
  size_t n = 0;
  const int64_t bytes[5] = {code_row, scale_row, code_row, scale_row, mass ? 4 * H : 0};
  for (const int64_t x : bytes) n += ((size_t)(batch * max_kept * x) + 255) & ~(size_t)255;
  return n;
}

hipError_t launch_paged_keep(const PagedKeepArgs& a, void* workspace, hipStream_t stream) {
  KeepLaunch l = keep_launch(a);
  if (a.to_table == nullptr && !through_workspace(a.batch, a.max_kept, a.code_row)) {
    Columns cols = {};
    int most = 1, at = 0;
    for (int i = 0; i < l.n_arrays; ++i) {
      const int lanes = i == 4 ? 1 : std::min(kMoveLanes, l.arrays[i].units);
      cols.first[i] = at;
      at += (l.arrays[i].units + lanes - 1) / lanes;
      most = std::max(most, lanes);
    }
    cols.first[l.n_arrays] = at;
    // threads for all entries at once, up to a workgroup's
    const int threads = (int)std::min<int64_t>(((int64_t)a.max_kept * most + 63) / 64 * 64, kMoveThreads);
    const dim3 grid((unsigned)at, (unsigned)a.batch);
    if (threads < kMoveThreads) keep_in_place_kernel<1, kMoveThreads><<<grid, threads, 0, stream>>>(a, l, cols);
    else keep_in_place_kernel<kMoveUnits, kMoveChunk><<<grid, threads, 0, stream>>>(a, l, cols);
    return hipGetLastError();
  }
  int64_t at = 0;
  l.staged = static_cast<uint8_t*>(workspace);
  for (int i = 0; i < l.n_arrays; ++i) {
    l.staged_at[i] = at;
    at += ((int64_t)a.batch * a.max_kept * l.arrays[i].units * l.arrays[i].unit + 255) & ~(int64_t)255;
  }
  const dim3 grid((unsigned)((a.max_kept + kRowsEach - 1) / kRowsEach), (unsigned)a.batch);
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
