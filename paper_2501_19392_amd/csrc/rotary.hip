// Rotary positions: the angles' tables, and rows of heads x 128 rotated by them.
#include "device_utils.h"
#include "kernels.h"

namespace aquakv {
namespace {

constexpr int kThreads = 256;

// ---------------------------------------------------------------- rows
// (x, y) -> (x c - y s, y c + x s) for the pairs of the first `dim` coordinates of a head: i and i + dim / 2 (halves), or 2 i and 2 i + 1.  A thread takes the same
// piece of kHeads heads of a token, for which it reads the angles once: with halves 16 bytes and the 16 bytes of their partners, with pairs 16 bytes.
// Bound by memory: 8192 tokens of 40 heads, 64 of 128 coordinates in pairs, 36.3 us, 4.7 TB/s (a copy of that size reaches 5.2).  One token of 40 heads: 3.0 us, a chain of
// two waits (position, angles) beside the row's own.
constexpr int kHeads = 4;
template <typename T, bool PAIRS>
__global__ __launch_bounds__(kThreads) void rotary_kernel(const RotaryArgs a) {
  constexpr int N = 16 / sizeof(T);                        // values of a piece
  constexpr int kAngles = PAIRS ? N / 2 : N;
  const int half = a.dim / 2, turned = PAIRS ? a.dim / N : half / N;      // pieces (pairs of pieces) of a head that are turned,
  const int pieces = turned + (a.in_place ? 0 : (kGroup - a.dim) / N);    // and those that are copied
  const int groups = (a.heads + kHeads - 1) / kHeads;
  const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t tg = id / pieces;
  const int piece = (int)(id - tg * pieces);
  const int64_t t = tg / groups;
  const int h0 = (int)(tg - t * groups) * kHeads;
  if (t >= a.tokens) return;
  const int pos = a.positions[t];
  const bool turn = piece < turned;
  const int at = turn ? piece * N : a.dim + (piece - turned) * N;
  const int64_t first = (int64_t)h0 * kGroup + at;         // (a row may pass 2^31 coordinates)
  const T* const x = static_cast<const T*>(a.x) + t * a.x_stride + first;
  T* const out = static_cast<T*>(a.out) + t * a.out_stride + first;
  float v[kHeads][N], w[kHeads][N];
#pragma unroll
  for (int k = 0; k < kHeads; ++k) {
    const int h = min(k, a.heads - 1 - h0);
    Storage<T>::load(x + h * kGroup, v[k]);
    if (!PAIRS && turn) Storage<T>::load(x + h * kGroup + half, w[k]);
  }
  if ((unsigned)pos >= (unsigned)a.rope_rows) return;      // (the row is left as it was)
  if (turn) {
    float c[kAngles], s[kAngles];
    const int64_t from = (int64_t)pos * half + (PAIRS ? at / 2 : at);
    if constexpr (kAngles >= 4) {
      load_f32(a.cos + from, c);
      load_f32(a.sin + from, s);
    } else {
#pragma unroll
      for (int i = 0; i < kAngles; ++i) { c[i] = a.cos[from + i]; s[i] = a.sin[from + i]; }
    }
#pragma unroll
    for (int k = 0; k < kHeads; ++k)
#pragma unroll
      for (int i = 0; i < kAngles; ++i) {
        float& lo = PAIRS ? v[k][2 * i % N] : v[k][i];
        float& hi = PAIRS ? v[k][(2 * i + 1) % N] : w[k][i];
        const float sn = a.transposed ? -s[i] : s[i], y = __fmaf_rn(lo, c[i], -(hi * sn));
        hi = __fmaf_rn(hi, c[i], lo * sn);
        lo = y;
      }
  }
#pragma unroll
  for (int k = 0; k < kHeads; ++k) {
    if (h0 + k >= a.heads) break;
    Storage<T>::template store<false>(out + k * kGroup, 0, v[k]);
    if (!PAIRS && turn) Storage<T>::template store<false>(out + k * kGroup + half, 0, w[k]);
  }
}

// ---------------------------------------------------------------- tables
// cos, sin of 2 pi x for x in turns, |x| <= 1 / 8 taken off the nearest quarter (both exact in 64 bits), in 32 bits from there: Taylor's series of an angle of
// at most pi / 4, up to terms of 2e-9 of the largest value.
__device__ __forceinline__ void cos_sin(double turns, float& c, float& s) {
  const double x = turns - __builtin_rint(turns), quarter = __builtin_rint(4.0 * x);
  const float y = (float)((x - 0.25 * quarter) * 6.283185307179586476925), z = y * y;
  const float sn = __fmaf_rn(y * z, __fmaf_rn(z, __fmaf_rn(z, __fmaf_rn(z, 1.0f / 362880, -1.0f / 5040), 1.0f / 120), -1.0f / 6), y);
  const float cs = __fmaf_rn(z, __fmaf_rn(z, __fmaf_rn(z, __fmaf_rn(z, __fmaf_rn(z, -1.0f / 3628800, 1.0f / 40320), -1.0f / 720), 1.0f / 24), -0.5f), 1.0f);
  const int q = (int)quarter & 3;
  c = (q & 1) ? sn : cs;
  s = (q & 1) ? cs : sn;
  if (q == 1 || q == 2) c = -c;
  if (q == 2 || q == 3) s = -s;
}
// A thread takes four neighbouring frequencies of kTableRows rows, `step` apart.  Bound by the stores: 131 072 x 64 angles 13.2 us, 5.1 TB/s.
// Fewer rows each where that leaves threads for the whole chip: 4096 x 64 angles 3.3 us, with 8 rows each 5.1.
constexpr int kTableRows = 8, kTableThreads = 1 << 16;
__global__ __launch_bounds__(kThreads) void rotary_tables_kernel(const RotaryTablesArgs a) {
  const int columns = a.pairs / 4, id = blockIdx.x * kThreads + threadIdx.x, column = id % columns;
  double f[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = a.turns[4 * column + i];
  int64_t row = id / columns;
#pragma unroll 1
  for (int k = 0; k < kTableRows && row < a.rows; ++k, row += a.step) {
    f32x4 c, s;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float cs, sn;
      cos_sin((double)(a.first + row) * f[i], cs, sn);
      c[i] = cs * a.magnitude;
      s[i] = sn * a.magnitude;
    }
    *reinterpret_cast<f32x4*>(a.cos + row * a.pairs + 4 * column) = c;
    *reinterpret_cast<f32x4*>(a.sin + row * a.pairs + 4 * column) = s;
  }
}

}  // namespace

hipError_t launch_rotary(int dtype, bool pairs, const RotaryArgs& a, hipStream_t stream) {
  const int n = dtype == kBF16 ? 8 : 4, turned = (pairs ? a.dim : a.dim / 2) / n, pieces = turned + (a.in_place ? 0 : (kGroup - a.dim) / n);
  const int64_t threads = a.tokens * ((a.heads + kHeads - 1) / kHeads) * pieces;
  const unsigned blocks = (unsigned)((threads + kThreads - 1) / kThreads);
  if (dtype == kBF16) {
    if (pairs) rotary_kernel<bf16_t, true><<<blocks, kThreads, 0, stream>>>(a);
    else rotary_kernel<bf16_t, false><<<blocks, kThreads, 0, stream>>>(a);
  } else {
    if (pairs) rotary_kernel<float, true><<<blocks, kThreads, 0, stream>>>(a);
    else rotary_kernel<float, false><<<blocks, kThreads, 0, stream>>>(a);
  }
  return hipGetLastError();
}

hipError_t launch_rotary_tables(const RotaryTablesArgs& args, hipStream_t stream) {
  RotaryTablesArgs a = args;
  const int64_t columns = a.pairs / 4;
  a.step = std::max((a.rows + kTableRows - 1) / kTableRows, std::min(a.rows, kTableThreads / columns));
  rotary_tables_kernel<<<(unsigned)((a.step * columns + kThreads - 1) / kThreads), kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace aquakv
