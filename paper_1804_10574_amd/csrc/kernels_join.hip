// Dropout from a counter-based generator, and the join of a residual branch: x = residual + dropout(y), out = gain * x * rstd with
// rstd = (mean x^2 + eps)^-1/2, its backward pass and its 8-bit output. All of it is bound by memory traffic.
//
// The draws: Philox4x32 with 7 rounds (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011; the fewest rounds that
// pass their statistical tests), a function of a 128-bit counter (column / 8, row, step) and a 64-bit key. A block's 128 bits are the draws of 8
// neighbouring columns, 16 bits each, compared with limit = round(65536 p): one block per 16-byte store, where 32-bit draws would take two
// and make the generator the bound. The kept share is then (65536 - limit) / 65536 exactly, and that is what kept elements are divided by.
// No mask is stored: whoever needs it again (a backward pass, the re-forward of a delayed iteration) passes the same seed and step.
#include "ddg_device.h"
#include "ddg_token.h"

namespace ddg {
namespace {

__device__ __forceinline__ void philox(uint32_t c0, uint32_t c1, const DropArgs& d, uint32_t (&o)[4]) {
  uint32_t c2 = d.step0, c3 = d.step1, k0 = d.key0, k1 = d.key1;
#pragma unroll
  for (int r = 0; r < 7; ++r) {
    const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
    c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
    c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
    c1 = (uint32_t)b; c3 = (uint32_t)a;
    k0 += 0x9E3779B9u; k1 += 0xBB67AE85u;
  }
  o[0] = c0; o[1] = c1; o[2] = c2; o[3] = c3;
}

// v of the 8 columns of unit `u` in row `row`, dropped or scaled
__device__ __forceinline__ void drop8(float (&v)[8], int row, int u, const DropArgs& d) {
  uint32_t w[4];
  philox((uint32_t)u, (uint32_t)row, d, w);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[2 * j] = (w[j] & 0xffffu) >= d.limit ? v[2 * j] * d.scale : 0.f;
    v[2 * j + 1] = (w[j] >> 16) >= d.limit ? v[2 * j + 1] * d.scale : 0.f;
  }
}

// 8 columns of a row, as they lie in memory. VEC: 16-byte pieces, and a row holds a whole number of them. Otherwise elements, those past `n` zero.
template <typename T, bool VEC> struct Unit {
  static constexpr int PIECES = 8 / Store<T>::VEC;
  typename Store<T>::vec_t v[PIECES];
  __device__ __forceinline__ void load(const T* p, int n) {
    if (VEC) {
#pragma unroll
      for (int i = 0; i < PIECES; ++i) v[i] = reinterpret_cast<const typename Store<T>::vec_t*>(p)[i];
    } else {
      T e[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) e[i] = i < n ? p[i] : T{};
      __builtin_memcpy(v, e, sizeof(v));
    }
  }
  __device__ __forceinline__ void zero() { __builtin_memset(v, 0, sizeof(v)); }
  __device__ __forceinline__ void get(float (&o)[8]) const {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      float t[Store<T>::VEC];
      Store<T>::unpack_vec(v[i], t);
#pragma unroll
      for (int j = 0; j < Store<T>::VEC; ++j) o[i * Store<T>::VEC + j] = t[j];
    }
  }
  __device__ static __forceinline__ void store(T* p, const float (&o)[8], int n) {
    if (VEC) {
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        float t[Store<T>::VEC];
#pragma unroll
        for (int j = 0; j < Store<T>::VEC; ++j) t[j] = o[i * Store<T>::VEC + j];
        Store<T>::store_vec(p + i * Store<T>::VEC, t);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) if (i < n) Store<T>::store1(p + i, o[i]);
    }
  }
};

// ---- dropout alone -------------------------------------------------------------------------------

template <typename T, bool VEC>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs a, int row0, int units, ImgOf per_row, int upr) {
  for (int q = blockIdx.x * 256 + threadIdx.x; q < units; q += gridDim.x * 256) {
    const int r = per_row.of(q), u = q - r * upr, row = row0 + r, n = a.cols - u * 8;
    Unit<T, VEC> in;
    in.load((const T*)a.x + (size_t)row * a.ld_x + u * 8, n);
    float v[8];
    in.get(v);
    if (a.drop.limit) drop8(v, row, u, a.drop);
    Unit<T, VEC>::store((T*)a.y + (size_t)row * a.ld_y + u * 8, v, n);
  }
}

// ---- the join ------------------------------------------------------------------------------------

__device__ __forceinline__ float wave_sum(float v) {
  v = row_sum16(v);
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}
__device__ __forceinline__ float row_max16(float v) {
  v = fmaxf(v, dpp_move<0xB1>(v));
  v = fmaxf(v, dpp_move<0x4E>(v));
  v = fmaxf(v, dpp_move<0x141>(v));
  return fmaxf(v, dpp_move<0x140>(v));
}
__device__ __forceinline__ float wave_max(float v) {
  v = row_max16(v);
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}
// Of all W waves of a row, in every lane; red: W floats of LDS, of its own for each use
template <int W> __device__ __forceinline__ float row_sum(float v, float* red) {
  v = wave_sum(v);
  if (W == 1) return v;
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  float t = 0.f;
#pragma unroll
  for (int i = 0; i < W; ++i) t += red[i];
  return t;
}
template <int W> __device__ __forceinline__ float row_max(float v, float* red) {
  v = wave_max(v);
  if (W == 1) return v;
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  float t = red[0];
#pragma unroll
  for (int i = 1; i < W; ++i) t = fmaxf(t, red[i]);
  return t;
}

__device__ __forceinline__ void gain8(const float* gain, int u, int n, float (&g)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) g[i] = gain && i < n ? gain[u * 8 + i] : 1.f;
}

// e4m3 of a pair, round to nearest even; values past 448 (the rounding of v * 448 / amax can pass it by a bit) become 448. NaN stays NaN.
__device__ __forceinline__ float clamp448(float v) { return v > 448.f ? 448.f : v < -448.f ? -448.f : v; }
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(clamp448(a), clamp448(b), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(clamp448(c), clamp448(d), w, true);
}

// A row is held by W waves, U units of 8 columns a lane, in registers: each operand is read once and each result written once.
// out comes from the x of 32 bits, not from the stored one: one rounding instead of two.
template <typename T, int W, int U, bool VEC, bool Q8>
__global__ __launch_bounds__(W == 1 ? 256 : W * 64) void join_forward_kernel(JoinArgs a) {
  constexpr int TPR = W * 64, RPB = W == 1 ? 4 : 1;
  __shared__ float red[2][W];
  const int lane = threadIdx.x % TPR, row = blockIdx.x * RPB + threadIdx.x / TPR;
  if (W == 1 && row >= a.rows) return;
  const int upr = (a.cols + 7) / 8;
  Unit<T, VEC> y[U], res[U];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int u = lane + i * TPR;
    y[i].zero(); res[i].zero();
    if (u < upr) {
      y[i].load((const T*)a.y + (size_t)row * a.ld_y + u * 8, a.cols - u * 8);
      if (a.residual) res[i].load((const T*)a.residual + (size_t)row * a.ld_residual + u * 8, a.cols - u * 8);
    }
  }
  float x[U][8], ss = 0.f;
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int u = lane + i * TPR;
    float r[8];
    y[i].get(x[i]);
    res[i].get(r);
    if (a.drop.limit) drop8(x[i], row, u, a.drop);
#pragma unroll
    for (int j = 0; j < 8; ++j) { x[i][j] += r[j]; ss += x[i][j] * x[i][j]; }
  }
  const float rstd = rsqrtf(row_sum<W>(ss, red[0]) / (float)a.cols + a.eps);
  if (a.rstd && lane == 0) a.rstd[row] = rstd;
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int u = lane + i * TPR, n = a.cols - u * 8;
    if (a.x && u < upr) Unit<T, VEC>::store((T*)a.x + (size_t)row * a.ld_x + u * 8, x[i], n);
    float g[8];
    gain8(a.gain, u, n, g);
#pragma unroll
    for (int j = 0; j < 8; ++j) { x[i][j] = x[i][j] * rstd * g[j]; top = fmaxf(top, fabsf(x[i][j])); }
    if (!Q8 && u < upr) Unit<T, VEC>::store((T*)a.out + (size_t)row * a.ld_out + u * 8, x[i], n);
  }
  if (!Q8) return;
  if (!a.group) top = row_max<W>(top, red[1]);
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int u = lane + i * TPR, n = a.cols - u * 8;
    float m = top;
    if (a.group) {               // 128 columns: the 16 lanes of a row of the wave
      m = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) m = fmaxf(m, fabsf(x[i][j]));
      m = row_max16(m);
    }
    const float scale = fmaxf(m / 448.f, 0x1p-126f);
    if (u >= upr) continue;
    if (a.group ? lane % 16 == 0 : lane == 0 && i == 0)
      a.scale[a.group ? (size_t)row * ((a.cols + 127) / 128) + u / 16 : (size_t)row] = scale;
    uint32_t w[2];
    w[0] = e4m3x4(x[i][0] / scale, x[i][1] / scale, x[i][2] / scale, x[i][3] / scale);
    w[1] = e4m3x4(x[i][4] / scale, x[i][5] / scale, x[i][6] / scale, x[i][7] / scale);
    uint8_t* q = a.q + (size_t)row * a.ld_out + u * 8;
    if (VEC) {
      *reinterpret_cast<uint2*>(q) = make_uint2(w[0], w[1]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) if (j < n) q[j] = (uint8_t)(w[j / 4] >> (8 * (j % 4)));
    }
  }
}

// With xhat = x rstd and c = mean(gain d_out xhat): d_residual = d_x + rstd (gain d_out - xhat c), d_y its dropped form, and a
// workgroup's rows of d_gain = sum d_out xhat in registers over all the rows that it takes, one row of `partial` in the end.
template <typename T, int W, int U, bool VEC>
__global__ __launch_bounds__(W == 1 ? 256 : W * 64) void join_backward_kernel(JoinArgs a) {
  constexpr int TPR = W * 64, RPB = W == 1 ? 4 : 1;
  __shared__ float red[2][W];
  __shared__ float joined[W == 1 ? 3 : 1][W == 1 ? U * 512 : 1];
  const int lane = threadIdx.x % TPR, part = threadIdx.x / TPR;
  const int upr = (a.cols + 7) / 8;
  float dg[U][8];
#pragma unroll
  for (int i = 0; i < U; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) dg[i][j] = 0.f;
  int turn = 0;
  for (int row = blockIdx.x * RPB + part; row < a.rows; row += gridDim.x * RPB, turn ^= 1) {
    Unit<T, VEC> xv[U], dv[U], sv[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = lane + i * TPR, n = a.cols - u * 8;
      xv[i].zero(); dv[i].zero(); sv[i].zero();
      if (u < upr) {
        xv[i].load((const T*)a.x + (size_t)row * a.ld_x + u * 8, n);
        dv[i].load((const T*)a.d_out + (size_t)row * a.ld_out + u * 8, n);
        if (a.d_x) sv[i].load((const T*)a.d_x + (size_t)row * a.ld_x + u * 8, n);
      }
    }
    const float rstd = a.rstd[row];
    float c = 0.f;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = lane + i * TPR;
      float x[8], d[8], g[8];
      xv[i].get(x); dv[i].get(d);
      gain8(a.gain, u, a.cols - u * 8, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float t = d[j] * (x[j] * rstd);
        dg[i][j] += t;
        c += t * g[j];
      }
    }
    c = row_sum<W>(c, red[turn]) / (float)a.cols;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = lane + i * TPR, n = a.cols - u * 8;
      float x[8], d[8], g[8], s[8];
      xv[i].get(x); dv[i].get(d); sv[i].get(s);
      gain8(a.gain, u, n, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] += rstd * (d[j] * g[j] - x[j] * rstd * c);
      if (u >= upr) continue;
      if (a.d_residual) Unit<T, VEC>::store((T*)a.d_residual + (size_t)row * a.ld_residual + u * 8, s, n);
      if (a.d_y) {
        if (a.drop.limit) drop8(s, row, u, a.drop);
        Unit<T, VEC>::store((T*)a.d_y + (size_t)row * a.ld_y + u * 8, s, n);
      }
    }
  }
  if (!a.d_gain) return;
  if (W == 1) {
    if (part) {
#pragma unroll
      for (int i = 0; i < U; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) joined[part - 1][(i * 8 + j) * 64 + lane] = dg[i][j];
    }
    __syncthreads();
    if (part) return;
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int q = 0; q < 3; ++q) dg[i][j] += joined[q][(i * 8 + j) * 64 + lane];
  }
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int u = lane + i * TPR, n = a.cols - u * 8;
#pragma unroll
    for (int j = 0; j < 8; ++j) if (u < upr && j < n) a.partial[(size_t)blockIdx.x * a.cols + u * 8 + j] = dg[i][j];
  }
}

// d_gain: the partial rows in order, four threads a column that take a quarter of them each
__global__ __launch_bounds__(256) void join_gain_kernel(const float* partial, int groups, int cols, float* d_gain) {
  __shared__ float red[256];
  const int c = blockIdx.x * 64 + threadIdx.x % 64, part = threadIdx.x / 64;
  const int per = (groups + 3) / 4, lo = part * per, hi = min(groups, lo + per);
  float t = 0.f;
  if (c < cols) {
#pragma unroll 16
    for (int r = lo; r < hi; ++r) t += partial[(size_t)r * cols + c];
  }
  red[threadIdx.x] = t;
  __syncthreads();
  if (part == 0 && c < cols) d_gain[c] = red[threadIdx.x] + red[threadIdx.x + 64] + red[threadIdx.x + 128] + red[threadIdx.x + 192];
}

bool aligned(const void* p, long ld, size_t size, size_t to) { return !p || ((uintptr_t)p % to == 0 && (size_t)ld * size % to == 0); }

template <typename T, int W, int U, bool VEC>
hipError_t forward_run(const JoinArgs& a, hipStream_t s) {
  const dim3 grid(W == 1 ? (a.rows + 3) / 4 : a.rows), block(W == 1 ? 256 : W * 64);
  if (a.q) DDG_LAUNCH((join_forward_kernel<T, W, U, VEC, true>), grid, block, 0, s, a);
  else DDG_LAUNCH((join_forward_kernel<T, W, U, VEC, false>), grid, block, 0, s, a);
  return hipGetLastError();
}
template <typename T, int W, int U, bool VEC>
hipError_t backward_run(const JoinArgs& a, hipStream_t s) {
  const int groups = join_groups(a.rows, a.cols);
  DDG_LAUNCH((join_backward_kernel<T, W, U, VEC>), dim3(groups), dim3(W == 1 ? 256 : W * 64), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.d_gain) return e;
  DDG_LAUNCH(join_gain_kernel, dim3((a.cols + 63) / 64), dim3(256), 0, s, a.partial, groups, a.cols, a.d_gain);
  return hipGetLastError();
}

// Waves a row and units a lane: the least registers that hold the row
template <typename T, bool VEC> hipError_t forward_any(const JoinArgs& a, hipStream_t s) {
  const int upr = (a.cols + 7) / 8;
  if (upr <= 64) return forward_run<T, 1, 1, VEC>(a, s);
  if (upr <= 256) return forward_run<T, 4, 1, VEC>(a, s);
  if (upr <= 512) return forward_run<T, 4, 2, VEC>(a, s);
  if (upr <= 1024) return forward_run<T, 4, 4, VEC>(a, s);
  return forward_run<T, 16, 4, VEC>(a, s);
}
template <typename T, bool VEC> hipError_t backward_any(const JoinArgs& a, hipStream_t s) {
  const int upr = (a.cols + 7) / 8;
  if (upr <= 64) return backward_run<T, 1, 1, VEC>(a, s);
  if (upr <= 256) return backward_run<T, 4, 1, VEC>(a, s);
  if (upr <= 512) return backward_run<T, 4, 2, VEC>(a, s);
  if (upr <= 1024) return backward_run<T, 4, 4, VEC>(a, s);
  return backward_run<T, 16, 4, VEC>(a, s);
}

}  // namespace

int join_groups(int rows, int cols) {
  const int upr = (cols + 7) / 8, per = upr <= 64 ? 4 : 1;
  const int most = upr <= 1024 ? 1024 : 512, want = (rows + per - 1) / per;
  return want < 1 ? 1 : want < most ? want : most;
}

hipError_t dropout_launch(const DropoutArgs& a, hipStream_t s) {
  const size_t size = dtype_size(a.dtype);
  const bool vec = a.cols % 8 == 0 && aligned(a.x, a.ld_x, size, 16) && aligned(a.y, a.ld_y, size, 16);
  const int upr = (a.cols + 7) / 8, most = (1 << 30) / upr;            // a launch takes up to 2^30 units
  for (int row0 = 0; row0 < a.rows; row0 += most) {
    const int units = (a.rows - row0 < most ? a.rows - row0 : most) * upr;
    const ImgOf per_row = ImgOf::make(upr, units);
    const int want = (units + 255) / 256;
    const dim3 grid(want < 8192 ? want : 8192);
    if (a.dtype == BF16) {
      if (vec) DDG_LAUNCH((dropout_kernel<bf16_t, true>), grid, dim3(256), 0, s, a, row0, units, per_row, upr);
      else DDG_LAUNCH((dropout_kernel<bf16_t, false>), grid, dim3(256), 0, s, a, row0, units, per_row, upr);
    } else {
      if (vec) DDG_LAUNCH((dropout_kernel<float, true>), grid, dim3(256), 0, s, a, row0, units, per_row, upr);
      else DDG_LAUNCH((dropout_kernel<float, false>), grid, dim3(256), 0, s, a, row0, units, per_row, upr);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t join_forward_launch(const JoinArgs& a, hipStream_t s) {
  const size_t size = dtype_size(a.dtype);
  const bool vec = a.cols % 8 == 0 && aligned(a.y, a.ld_y, size, 16) && aligned(a.residual, a.ld_residual, size, 16) &&
                   aligned(a.x, a.ld_x, size, 16) && (a.q ? aligned(a.q, a.ld_out, 1, 8) : aligned(a.out, a.ld_out, size, 16));
  if (a.dtype == BF16) return vec ? forward_any<bf16_t, true>(a, s) : forward_any<bf16_t, false>(a, s);
  return vec ? forward_any<float, true>(a, s) : forward_any<float, false>(a, s);
}

hipError_t join_backward_launch(const JoinArgs& a, hipStream_t s) {
  const size_t size = dtype_size(a.dtype);
  const bool vec = a.cols % 8 == 0 && aligned(a.x, a.ld_x, size, 16) && aligned(a.d_out, a.ld_out, size, 16) && aligned(a.d_x, a.ld_x, size, 16) &&
                   aligned(a.d_residual, a.ld_residual, size, 16) && aligned(a.d_y, a.ld_y, size, 16);
  if (a.dtype == BF16) return vec ? backward_any<bf16_t, true>(a, s) : backward_any<bf16_t, false>(a, s);
  return vec ? backward_any<float, true>(a, s) : backward_any<float, false>(a, s);
}

}  // namespace ddg
