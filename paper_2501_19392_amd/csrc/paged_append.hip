// New tokens of a cache that lives in pages of codes: keys rotated to their positions, keys and values quantized (Sect. 2 of the AQUA-KV
// paper; no predictors), codes and scales to the rows `slots` names.  One launch for both tensors.
//
// A head's 128 values are held by eight lanes x 16 as in the stand-alone quantizer, whose body this is: the rotary embedding pairs
// coordinates 64 apart, which sit in the same register of the lane whose position differs in the uppermost bit.
//
// Bound by the vector pipes and LDS: 8192 tokens of 8 heads, 256 points, with the rows read back, take 33.7 us (80 MB at 2.4 TB/s) and 840 instructions
// for 16 values of a lane, 82 % of the cycles; the rotations there and back are 224 of them, the search 280.  LDS is busy in 81 % of the cycles with the search's
// look-ups, 58 % of that for bank conflicts.  Uniform codes, which have neither, are bound by memory (15.5 us, at a copy's rate).  A few tokens are one chain of waits (arguments,
// rows and tables, grid and search table to LDS, barrier, rotation, search): one token 5.0 us in a trace (a call in a graph 6.0, with
// uniform codes, which stage nothing, 3.3).  What came out no faster: rows of a round requested during the one before
// (36.2 us, for registers); 32 values a lane in columns, with the way back on the matrix cores and the grid 16 times in LDS, which takes
// bank conflicts from 58 to 22 % of the LDS cycles (34.5 us: 15 % fewer instructions, and 6 more of 64 KB to fill; one token 7.9).
#include "codec_core.h"
#include "kernels.h"

namespace aquakv {
namespace {

constexpr int kThreads = 256;
constexpr int N = 16, kLanes = kGroup / N, kGroups = kThreads / kLanes;      // values per lane, lanes per head group, groups per round

// blockIdx.y: keys, values.  Rows whose slot or position lies outside are left out: nothing is written for them.
template <typename T, int NCW>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(4))) void paged_append_kernel(const PagedAppendArgs a) {
  const bool keys = blockIdx.y == 0;
  const T* const X = static_cast<const T*>(keys ? a.K : a.V);
  const int64_t x_stride = keys ? a.k_stride : a.v_stride;
  T* const Xhat = static_cast<T*>(keys ? a.Khat : a.Vhat);
  uint8_t* const codes = keys ? a.pool.k_codes : a.pool.v_codes;
  uint16_t* const scales = keys ? a.pool.k_scales : a.pool.v_scales;
  const int8_t* const signs = keys ? a.signs_k : a.signs_v;
  const bool rope = keys && a.rope_cos != nullptr;
  __shared__ Lds lds;
  const int l = group_pos<N>(threadIdx.x), slot_in_block = threadIdx.x / kLanes;
  const unsigned n_groups = (unsigned)a.tokens * (unsigned)a.H, step = gridDim.x * kGroups;
  float v[N];
  int64_t row;
  int pos = 0;
  const auto request = [&](unsigned g0) {
    const unsigned gid = min(g0 + slot_in_block, n_groups - 1), t = gid / (unsigned)a.H;      // (every lane stays in the DPP exchanges)
    row = a.slots[t];
    if (a.rope_cos != nullptr) pos = a.positions[t];
    Storage<T>::load(X + t * x_stride + (gid - t * (unsigned)a.H) * kGroup + l * N, v);
  };
  request(blockIdx.x * kGroups);                          // on the way while the tables are (one token 5.5 us a call in a graph, behind them 5.7)
  if constexpr (!is_rtn(NCW)) {
    TableRegs<kThreads> table_regs;
    if (a.table != nullptr) table_regs.request(a.table);
    load_codebook<NCW>(a.codebook, lds.cb);
    if (a.table != nullptr) table_regs.store(lds.table);
    __syncthreads();
  }
  for (unsigned g0 = blockIdx.x * kGroups;;) {
    const unsigned gid = min(g0 + slot_in_block, n_groups - 1), head = gid % (unsigned)a.H;
    bool active = g0 + slot_in_block < n_groups && (uint64_t)row < (uint64_t)a.pool.rows;
    if (a.rope_cos != nullptr && (unsigned)pos >= (unsigned)a.rope_rows) { active = false; pos = 0; }      // (a token is left out as a whole)
    float sf[N] = {};
    if constexpr (!is_rtn(NCW)) load_signs(signs, (int)head, l, sf);
    if (rope) rope128(v, l, a.rope_cos + (int64_t)pos * (kGroup / 2), a.rope_sin + (int64_t)pos * (kGroup / 2));
    quantize_residual<NCW>(v, sf, l, lds.cb, a.table != nullptr ? lds.table : nullptr, active, row * a.H + head, codes, scales, Xhat != nullptr);
    if (Xhat != nullptr) {
      const float zero[N] = {};
      finish_hat<NCW>(v, sf, zero);
      if (active) Storage<T>::template store<false>(Xhat + (int64_t)gid * kGroup, l, v);
    }
    if ((g0 += step) >= n_groups) break;
    request(g0);
  }
}

}  // namespace

hipError_t launch_paged_append(int dtype, int n_codewords, const PagedAppendArgs& a, hipStream_t stream) {
  const int64_t blocks = (a.tokens * a.H + kGroups - 1) / kGroups;
  const dim3 grid((unsigned)(blocks < 512 ? blocks : 512), 2);
#define AQUAKV_APPEND(T, NCW) paged_append_kernel<T, NCW><<<grid, kThreads, 0, stream>>>(a)
#define AQUAKV_APPEND_T(T)                                    \
  switch (n_codewords) {                                      \
    case kRtn2: AQUAKV_APPEND(T, kRtn2); break;               \
    case kRtn4: AQUAKV_APPEND(T, kRtn4); break;               \
    case 16: AQUAKV_APPEND(T, 16); break;                     \
    case 64: AQUAKV_APPEND(T, 64); break;                     \
    default: AQUAKV_APPEND(T, 256);                           \
  }
  if (dtype == kBF16) { AQUAKV_APPEND_T(bf16_t) } else { AQUAKV_APPEND_T(float) }
#undef AQUAKV_APPEND_T
#undef AQUAKV_APPEND
  return hipGetLastError();
}

}  // namespace aquakv
