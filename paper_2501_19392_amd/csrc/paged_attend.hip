// Attention over a cache that lives in pages of codes (4 bits and the framework's other widths), read as they are: no row is recovered.
// With the rotation R = H S / sqrt(128) of the quantizer (Sect. 2 of the AQUA-KV paper) a key is R^T (sigma C[codes]), so
//   q . khat = sigma (R q) . C[codes],      sum_t p_t vhat_t = R^T sum_t (p_t sigma_t) C[codes_t]:
// the query is rotated once, the result once, and in between a code is a look-up.  (Uniform backbone: no rotation, (code - zero) step.)
//
// One wave per query head of a query: a lane takes a token of 64 for the scores, two coordinates for the values.
#include "codec_core.h"
#include "kernels.h"

namespace aquakv {
namespace {

// What a sequence asks: `count` queries, its last tokens, rows first ... of q, of which n are answered; len tokens are cached.
struct PagedQueries { int64_t first; int count, n, len; };
__device__ __forceinline__ PagedQueries paged_queries(const PagedAttendArgs& a, int b) {
  PagedQueries w;
  w.first = (int64_t)b * a.max_queries;
  w.count = a.max_queries;
  if (a.q_start != nullptr) {
    const int64_t from = a.q_start[b], to = a.q_start[b + 1];
    w.first = from < 0 ? 0 : from < a.q_rows ? from : a.q_rows;
    const int64_t end = to < w.first ? w.first : to < a.q_rows ? to : a.q_rows;
    w.count = (int)(end - w.first);
  }
  w.n = min(w.count, a.max_queries);
  const int64_t room = (int64_t)a.table_pages * a.pool.page_tokens;
  w.len = (int)min((int64_t)max(a.seq_lens[b], 0), room);
  return w;
}

template <int NCW> __device__ __forceinline__ float2 pair_of(const uint8_t* __restrict__ row, int i, const float2* cb) {
  constexpr int c = CodeBits<NCW>::c;
  const int bit = c * i;
  uint32_t w = row[bit >> 3];
  if constexpr (c == 6) { if ((bit & 7) > 2) w |= (uint32_t)row[(bit >> 3) + 1] << 8; }
  const uint32_t code = (w >> (bit & 7)) & ((1u << c) - 1u);
  if constexpr (is_rtn(NCW)) return make_float2((float)(code & ((1u << NCW) - 1u)), (float)(code >> NCW));
  else return cb[code];
}

// rotated coordinates 2 lane, 2 lane + 1 of a vector whose coordinates 2 lane, 2 lane + 1 are (x, y)
__device__ __forceinline__ void wht_wave(float& x, float& y, int lane) {
  const float s = x + y, d = x - y;
  x = s; y = d;
  for (int m = 1; m < 64; m <<= 1) {
    const float px = __shfl_xor(x, m), py = __shfl_xor(y, m);
    x = (lane & m) ? px - x : x + px;
    y = (lane & m) ? py - y : y + py;
  }
}

template <typename T, int NCW>
__global__ __launch_bounds__(64) void paged_attend_kernel(const PagedAttendArgs a) {
  __shared__ float2 cb[is_rtn(NCW) ? 1 : NCW];
  __shared__ float qs[kGroup];
  const int lane = threadIdx.x, b = blockIdx.y, qi = blockIdx.x / a.q_heads, qh = blockIdx.x % a.q_heads, h = qh / (a.q_heads / a.H);
  if constexpr (!is_rtn(NCW))
    for (int j = lane; j < NCW; j += 64) cb[j] = make_float2(a.codebook[2 * j], a.codebook[2 * j + 1]);
  const PagedQueries w = paged_queries(a, b);
  if (qi >= w.n) return;
  const int64_t qrow = w.first + qi;
  const int last = w.len - w.count + qi;                  // position of this query
  const T* const q = static_cast<const T*>(a.q) + qrow * a.q_stride + qh * kGroup;
  float x = (float)q[2 * lane], y = (float)q[2 * lane + 1];
  if constexpr (!is_rtn(NCW)) {
    x *= a.signs_k[h * kGroup + 2 * lane]; y *= a.signs_k[h * kGroup + 2 * lane + 1];
    wht_wave(x, y, lane);
    x *= kRsqrtG; y *= kRsqrtG;
  }
  qs[2 * lane] = x * a.scale; qs[2 * lane + 1] = y * a.scale;
  __syncthreads();
  constexpr int kRow = kGroup / 2 * CodeBits<NCW>::c / 8;
  float m = -INFINITY, sum = 0.f, ox = 0.f, oy = 0.f;
  for (int t0 = 0; t0 <= last; t0 += 64) {
    const int t = t0 + lane;
    int64_t gid = -1;
    if (t <= last) {
      const int page = a.page_table[(int64_t)b * a.table_pages + t / a.pool.page_tokens];
      if ((unsigned)page < (unsigned)a.pool.n_pages) gid = ((int64_t)page * a.pool.page_tokens + t % a.pool.page_tokens) * a.H + h;
    }
    float s = -INFINITY;
    if (gid >= 0) {
      float acc[2] = {0.f, 0.f};
      float zero[2] = {0.f, 0.f}, step[2];
      if constexpr (is_rtn(NCW)) {
        for (int k = 0; k < 2; ++k) {
          step[k] = half_bits_to_float(a.pool.k_scales[(gid * 2 + k) * 2]);
          zero[k] = (float)a.pool.k_scales[(gid * 2 + k) * 2 + 1];
        }
      } else {
        step[0] = step[1] = half_bits_to_float(a.pool.k_scales[gid]);
      }
      for (int i = 0; i < 64; ++i) {
        const float2 c = pair_of<NCW>(a.pool.k_codes + gid * kRow, i, cb);
        acc[i >> 5] += qs[2 * i] * (c.x - zero[i >> 5]) + qs[2 * i + 1] * (c.y - zero[i >> 5]);
      }
      s = acc[0] * step[0] + acc[1] * step[1];
    }
    float top = s;
    for (int k = 1; k < 64; k <<= 1) top = fmaxf(top, __shfl_xor(top, k));
    if (top == -INFINITY) continue;
    const float M = fmaxf(m, top), keep = expf(m - M), p = expf(s - M);
    float part = p;
    for (int k = 1; k < 64; k <<= 1) part += __shfl_xor(part, k);
    sum = sum * keep + part; ox *= keep; oy *= keep; m = M;
    for (int k = 0; k < 64; ++k) {
      const float pk = __shfl(p, k);
      const int64_t gk = __shfl(gid, k);
      if (gk < 0) continue;
      float zero = 0.f, step;
      if constexpr (is_rtn(NCW)) {
        step = half_bits_to_float(a.pool.v_scales[(gk * 2 + (lane >> 5)) * 2]);
        zero = (float)a.pool.v_scales[(gk * 2 + (lane >> 5)) * 2 + 1];
      } else {
        step = half_bits_to_float(a.pool.v_scales[gk]);
      }
      const float2 c = pair_of<NCW>(a.pool.v_codes + gk * kRow, lane, cb);
      ox += pk * step * (c.x - zero); oy += pk * step * (c.y - zero);
    }
  }
  const float inv = sum > 0.f ? 1.f / sum : 0.f;          // (no token: 0)
  ox *= inv; oy *= inv;
  if constexpr (!is_rtn(NCW)) {
    wht_wave(ox, oy, lane);
    ox *= kRsqrtG * a.signs_v[h * kGroup + 2 * lane]; oy *= kRsqrtG * a.signs_v[h * kGroup + 2 * lane + 1];
  }
  T* const out = static_cast<T*>(a.out) + (qrow * a.q_heads + qh) * kGroup;
  out[2 * lane] = (T)ox; out[2 * lane + 1] = (T)oy;
}

}  // namespace

hipError_t launch_paged_attend(int dtype, int n_codewords, const PagedAttendArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)(a.max_queries * a.q_heads), (unsigned)a.batch);
#define AQUAKV_ATTEND(T, NCW) paged_attend_kernel<T, NCW><<<grid, 64, 0, stream>>>(a)
#define AQUAKV_ATTEND_T(T)                                    \
  switch (n_codewords) {                                      \
    case kRtn2: AQUAKV_ATTEND(T, kRtn2); break;               \
    case kRtn4: AQUAKV_ATTEND(T, kRtn4); break;               \
    case 16: AQUAKV_ATTEND(T, 16); break;                     \
    case 64: AQUAKV_ATTEND(T, 64); break;                     \
    default: AQUAKV_ATTEND(T, 256);                           \
  }
  if (dtype == kBF16) { AQUAKV_ATTEND_T(bf16_t) } else { AQUAKV_ATTEND_T(float) }
#undef AQUAKV_ATTEND_T
#undef AQUAKV_ATTEND
  return hipGetLastError();
}

}  // namespace aquakv
