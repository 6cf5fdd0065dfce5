// Rotary positions: the pairs (a, b) of a head's first `rot` columns are turned by an angle that grows with the row's position,
//   (a cos - b sin, b cos + a sin) * magnitude,   angle = position * theta_i,
// backwards for the gradient. Pairs are neighbours (2i, 2i+1) or halves (i, i + rot/2).
// The angle: a table holds theta_i / 2 pi as a 64-bit fraction of a turn, so position times that, modulo 2^64, is the exact fraction of the last turn for the table's theta_i (within four
// steps of the true one: |position| 2^-62 of a turn), and fp32 takes what is left of a quarter to 2^-28: a position
// of a million radians is as good as one of one (in fp32 that product alone is off by 0.03 radians, in 64-bit floating point it costs more than the rows do).
// A workgroup forms the cosines and sines of its rows once, in LDS, for all heads. Bound by memory: 8192 rows of 40 heads of 128 in bf16 take 26 us (168 MB, 6.4 TB/s).
#include "ddg_mixing.h"
#include "ddg_rows.h"

namespace ddg {
namespace {

// Cosine and sine of `f` of 2^64 turns: the nearest quarter turn and what is left, at most an eighth either way, whose conversion keeps 24 bits
__device__ __forceinline__ float2 turn(uint64_t f) {
  const uint32_t quarter = (uint32_t)((f + (1ull << 61)) >> 62);
  const int64_t left = (int64_t)(f - ((uint64_t)quarter << 62));
  float s, c;
  sincospif((float)left * 0x1p-63f, &s, &c);
  const float a = quarter & 1 ? -s : c, b = quarter & 1 ? c : s;
  return quarter & 2 ? make_float2(-a, -b) : make_float2(a, b);
}

// n elements from p on, zeros behind them
template <typename T, bool VEC> __device__ __forceinline__ void get(const T* p, int n, float (&o)[Store<T>::VEC]) {
  constexpr int W = Store<T>::VEC;
  if (VEC || n >= W) {
    typename Store<T>::vec_t v;
    if (VEC) v = *reinterpret_cast<const typename Store<T>::vec_t*>(p);
    else __builtin_memcpy(&v, p, sizeof(v));
    Store<T>::unpack_vec(v, o);
  } else {
#pragma unroll
    for (int i = 0; i < W; ++i) o[i] = i < n ? Store<T>::load1(p + i) : 0.f;
  }
}
template <typename T, bool VEC> __device__ __forceinline__ void put(T* p, int n, const float (&o)[Store<T>::VEC], bool past) {
  constexpr int W = Store<T>::VEC;
  if (VEC || n >= W) {
    typename Store<T>::vec_t v;
    Store<T>::store_vec(reinterpret_cast<T*>(&v), o);
    if (VEC) put16(reinterpret_cast<typename Store<T>::vec_t*>(p), v, past);
    else __builtin_memcpy(p, &v, sizeof(v));
  } else {
#pragma unroll
    for (int i = 0; i < W; ++i) if (i < n) Store<T>::store1(p + i, o[i]);
  }
}

// RB rows a workgroup. A unit is 16 bytes of neighbouring pairs, or two of halves, or 16 bytes that are copied. VEC: every piece is whole and on its boundary.
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a, int RB, int turned, int copied, bool past, ImgOf per_row, ImgOf per_head, ImgOf pairs) {
  constexpr int W = Store<T>::VEC;
  extern __shared__ float2 turns[];                // [RB][rot / 2]
  const int half = a.rot / 2, row0 = blockIdx.x * RB, rows = min(RB, a.rows - row0);
  for (int i = threadIdx.x; i < rows * half; i += 256) {
    const int r = pairs.of(i), p = i - r * half;
    const int64_t pos = a.first + (a.positions ? a.positions[row0 + r] : row0 + r);
    float2 t = turn((uint64_t)pos * a.table[p]);
    if (a.inverse) t.y = -t.y;
    turns[i] = make_float2(t.x * a.magnitude, t.y * a.magnitude);
  }
  __syncthreads();
  const int units = turned + copied, upr = a.heads * units;
  for (int i = threadIdx.x; i < rows * upr; i += 256) {
    const int r = per_row.of(i), in_row = i - r * upr, head = per_head.of(in_row), u = in_row - head * units;
    const T* x = (const T*)a.x + (size_t)(row0 + r) * a.ld_x + head * a.dim;
    T* y = (T*)a.y + (size_t)(row0 + r) * a.ld_y + head * a.dim;
    const float2* t = turns + r * half;
    if (u >= turned) {
      const int c = a.rot + (u - turned) * W;
      float v[W];
      get<T, VEC>(x + c, a.dim - c, v);
      put<T, VEC>(y + c, a.dim - c, v, past);
    } else if (a.interleaved) {
      const int c = u * W;
      float v[W], o[W];
      get<T, VEC>(x + c, a.rot - c, v);
#pragma unroll
      for (int j = 0; j < W; j += 2) {
        const float2 w = VEC || c + j < a.rot ? t[(c + j) / 2] : make_float2(0.f, 0.f);
        o[j] = v[j] * w.x - v[j + 1] * w.y;
        o[j + 1] = v[j + 1] * w.x + v[j] * w.y;
      }
      put<T, VEC>(y + c, a.rot - c, o, past);
    } else {
      const int c = u * W, n = half - c;
      float v[W], h[W], o[W], p[W];
      get<T, VEC>(x + c, n, v);
      get<T, VEC>(x + half + c, n, h);
#pragma unroll
      for (int j = 0; j < W; ++j) {
        const float2 w = VEC || j < n ? t[c + j] : make_float2(0.f, 0.f);
        o[j] = v[j] * w.x - h[j] * w.y;
        p[j] = h[j] * w.x + v[j] * w.y;
      }
      put<T, VEC>(y + c, n, o, past);
      put<T, VEC>(y + half + c, n, p, past);
    }
  }
}

// One workgroup of 256 threads a row: a launch holds fewer than 2^32 threads
constexpr int ROWS_A_LAUNCH = 1 << 23;

template <typename T> hipError_t run(const RotaryArgs& a, hipStream_t s) {
  constexpr int W = Store<T>::VEC;
  const int half = a.rot / 2, span = a.interleaved ? a.rot : half;
  const int turned = (span + W - 1) / W, copied = a.x == a.y ? 0 : (a.dim - a.rot + W - 1) / W;
  const bool vec = span % W == 0 && a.dim % W == 0 && a.rot % W == 0 && aligned(a.x, a.ld_x, sizeof(T), 16) && aligned(a.y, a.ld_y, sizeof(T), 16);
  const int upr = a.heads * (turned + copied);
  const int rows = a.rows < ROWS_A_LAUNCH ? a.rows : ROWS_A_LAUNCH;
  // a workgroup has work for its threads, and the chip for all of them (8192 rows of 320 units: 34 us with one row, 38 with eight)
  int RB = 1;
  while (RB < 32 && RB * upr < 256 && RB * 512 <= rows && RB * 2 * half <= 1024) RB *= 2;
  const bool past = (size_t)a.rows * a.heads * a.dim * sizeof(T) > CACHED;
  const ImgOf per_row = ImgOf::make(upr, (long)RB * upr), per_head = ImgOf::make(turned + copied, upr), pairs = ImgOf::make(half, RB * half);
  const size_t lds = (size_t)RB * half * sizeof(float2);
  for (int row0 = 0; row0 < a.rows; row0 += ROWS_A_LAUNCH) {
    RotaryArgs b = a;
    b.x = (const T*)a.x + (size_t)row0 * a.ld_x;
    b.y = (T*)a.y + (size_t)row0 * a.ld_y;
    if (a.positions) b.positions = a.positions + row0;
    else b.first = a.first + row0;
    b.rows = a.rows - row0 < ROWS_A_LAUNCH ? a.rows - row0 : ROWS_A_LAUNCH;
    const dim3 grid((b.rows + RB - 1) / RB);
    if (vec) DDG_LAUNCH((rotary_kernel<T, true>), grid, dim3(256), lds, s, b, RB, turned, copied, past, per_row, per_head, pairs);
    else DDG_LAUNCH((rotary_kernel<T, false>), grid, dim3(256), lds, s, b, RB, turned, copied, past, per_row, per_head, pairs);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t rotary_launch(const RotaryArgs& a, hipStream_t s) { return a.dtype == BF16 ? run<bf16_t>(a, s) : run<float>(a, s); }

}  // namespace ddg
