// Dropout from a counter-based generator, and the join of a residual branch: x = residual + dropout(y), out = gain * x * rstd with
// rstd = (mean x^2 + eps)^-1/2, its backward pass and its 8-bit output. All of it is bound by memory traffic; on tensors that the last cache does not hold,
// 8192 x 2048 in bf16 takes 29 us forward (134 MB, 4.6 TB/s) and 38 us backward (168 MB, 4.5 TB/s), dropout of 8192 x 4096 24.6 us (134 MB, 5.5 TB/s); a copy
// reaches 5.2 to 5.4 TB/s there. A call of one row is its launch: 2.5 us of the device, 4 to 5 us of the host.
//
// The draws: Philox4x32 with 7 rounds (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011; the fewest rounds that
// pass their statistical tests), a function of a 128-bit counter (column / 8, row, step) and a 64-bit key. A block's 128 bits are the draws of 8
// neighbouring columns, 16 bits each, compared with limit = round(65536 p): one block per 16-byte store, where 32-bit draws would take two
// and make the generator the bound. The kept share is then (65536 - limit) / 65536 exactly, and that is what kept elements are divided by.
// No mask is stored: whoever needs it again (a backward pass, the re-forward of a delayed iteration) passes the same seed and step.
#include "ddg_rows.h"
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

// ---- dropout alone -------------------------------------------------------------------------------

// A 16-byte piece (fp32: two) a thread and trip; the draws' 14 products of 32 bits cost less than its loads and stores
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

// e4m3 of a pair, round to nearest even. Values past 448 (the rounding of v * 448 / amax can pass it by a bit) become 448. NaN stays NaN.
__device__ __forceinline__ float clamp448(float v) { return v > 448.f ? 448.f : v < -448.f ? -448.f : v; }
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(clamp448(a), clamp448(b), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(clamp448(c), clamp448(d), w, true);
}

// The longest rows leave no registers for the next row's operands or the gain: those are read when they are needed
template <int W, int U> constexpr bool LONGEST = W == 16 && U == 4;

// A row is held by W waves, U units of 8 columns a lane, in registers: each operand is read once and each result written once. A workgroup takes
// several rows, the next one's operands in flight while it works on one (8192 x 2048 in bf16: 24.7 us instead of 42.4 with a workgroup a row, whose gain came
// from the cache for every row, as many bytes as y). out comes from the x of 32 bits, not from the stored one: one rounding. Q8: the quotient by the scale is the rounded product
// with its reciprocal and one step from there by what it leaves over, which is the correctly rounded quotient (what is left over is exact for scales from 2^-93 on); the product
// alone puts a value next to a tie, one in some millions, to the other neighbour. (8192 x 2048 in bf16:
// 27.3-27.7 us, the product alone 27.0, a division 29.7.)
template <typename T, int W, int U, bool VEC, bool Q8>
__global__ __launch_bounds__(W == 1 ? 256 : W * 64) void join_forward_kernel(JoinArgs a) {
  constexpr int TPR = W * 64, RPB = W == 1 ? 4 : 1;
  constexpr bool AHEAD = !LONGEST<W, U>;
  __shared__ float red[2][2][W];
  const int lane = threadIdx.x % TPR, upr = (a.cols + 7) / 8, step = gridDim.x * RPB;
  int row = blockIdx.x * RPB + threadIdx.x / TPR;
  Unit<T, VEC> y[U], res[U];
  auto request = [&](int r) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = lane + i * TPR;
      if (u < upr) {
        y[i].load((const T*)a.y + (size_t)r * a.ld_y + u * 8, a.cols - u * 8);
        if (a.residual) res[i].load((const T*)a.residual + (size_t)r * a.ld_residual + u * 8, a.cols - u * 8);
      }
    }
  };
#pragma unroll
  for (int i = 0; i < U; ++i) { y[i].zero(); res[i].zero(); }
  if (AHEAD && row < a.rows) request(row);
  float g[U][8];
  if (AHEAD) load_gain<U, TPR>(a.gain, lane, a.cols, g);
  const float inv = 1.f / (float)a.cols;
  for (int turn = 0; row < a.rows; row += step, turn ^= 1) {
    if (!AHEAD) request(row);
    float x[U][8], ss = 0.f;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      float r[8];
      y[i].get(x[i]);
      res[i].get(r);
      if (a.drop.limit) drop8(x[i], row, lane + i * TPR, a.drop);
#pragma unroll
      for (int j = 0; j < 8; ++j) { x[i][j] += r[j]; ss += x[i][j] * x[i][j]; }
    }
    if (AHEAD && row + step < a.rows) request(row + step);
    const float rstd = rsqrtf(row_sum<W>(ss, red[turn][0]) * inv + a.eps);
    if (a.rstd && lane == 0) a.rstd[row] = rstd;
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = lane + i * TPR, n = a.cols - u * 8;
      if (a.x && u < upr) Unit<T, VEC>::store((T*)a.x + (size_t)row * a.ld_x + u * 8, x[i], n);
      if (!AHEAD) load_gain<1, TPR>(a.gain, u, a.cols, reinterpret_cast<float(&)[1][8]>(g[i]));
#pragma unroll
      for (int j = 0; j < 8; ++j) { x[i][j] = x[i][j] * rstd * g[i][j]; if (Q8) top = fmaxf(top, fabsf(x[i][j])); }
      if (!Q8 && u < upr) Unit<T, VEC>::store((T*)a.out + (size_t)row * a.ld_out + u * 8, x[i], n);
    }
    if (!Q8) continue;
    if (!a.group) top = row_max<W>(top, red[turn][1]);
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
      const float scale = fmaxf(m * (1.f / 448.f), 0x1p-126f), to = 1.f / scale;
      const auto over = [&](float v) { const float near = v * to; return fmaf(-fmaf(near, scale, -v), to, near); };     // (-0 stays -0)
      if (u >= upr) continue;
      if (a.group ? lane % 16 == 0 : lane == 0 && i == 0)
        a.scale[a.group ? (size_t)row * ((a.cols + 127) / 128) + u / 16 : (size_t)row] = scale;
      uint32_t w[2];
      w[0] = e4m3x4(over(x[i][0]), over(x[i][1]), over(x[i][2]), over(x[i][3]));
      w[1] = e4m3x4(over(x[i][4]), over(x[i][5]), over(x[i][6]), over(x[i][7]));
      uint8_t* q = a.q + (size_t)row * a.ld_out + u * 8;
      if (VEC) {
        *reinterpret_cast<uint2*>(q) = make_uint2(w[0], w[1]);
      } else if (n >= 8) {
        __builtin_memcpy(q, w, 8);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) if (j < n) q[j] = (uint8_t)(w[j / 4] >> (8 * (j % 4)));
      }
    }
  }
}

// With xhat = x rstd and c = mean(gain d_out xhat): d_residual = d_x + rstd (gain d_out - xhat c), d_y its dropped form, and a
// workgroup's rows of d_gain = sum d_out xhat in registers over all the rows that it takes, one row of `partial` in the end: no atomics, so the bits do not
// depend on the order of workgroups.
template <typename T, int W, int U, bool VEC>
__global__ __launch_bounds__(W == 1 ? 256 : W * 64) void join_backward_kernel(JoinArgs a) {
  constexpr int TPR = W * 64, RPB = W == 1 ? 4 : 1;
  constexpr bool AHEAD = !LONGEST<W, U>;
  __shared__ float red[2][W];
  __shared__ float joined[W == 1 ? 3 : 1][W == 1 ? U * 512 : 1];
  const int lane = threadIdx.x % TPR, part = threadIdx.x / TPR, step = gridDim.x * RPB;
  const int upr = (a.cols + 7) / 8;
  Unit<T, VEC> xv[U], dv[U], sv[U];
  float rstd = 0.f;
  auto request = [&](int r) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = lane + i * TPR, n = a.cols - u * 8;
      if (u < upr) {
        xv[i].load((const T*)a.x + (size_t)r * a.ld_x + u * 8, n);
        dv[i].load((const T*)a.d_out + (size_t)r * a.ld_out + u * 8, n);
        if (AHEAD && a.d_x) sv[i].load((const T*)a.d_x + (size_t)r * a.ld_x + u * 8, n);
      }
    }
    rstd = a.rstd[r];
  };
  float dg[U][8], g[U][8];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    xv[i].zero(); dv[i].zero(); sv[i].zero();
#pragma unroll
    for (int j = 0; j < 8; ++j) dg[i][j] = 0.f;
  }
  int row = blockIdx.x * RPB + part;
  if (AHEAD && row < a.rows) request(row);
  if (AHEAD) load_gain<U, TPR>(a.gain, lane, a.cols, g);
  const float inv = 1.f / (float)a.cols;
  for (int turn = 0; row < a.rows; row += step, turn ^= 1) {
    if (!AHEAD) request(row);
    float x[U][8], d[U][8], s[U][8], c = 0.f;
    const float by = rstd;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      xv[i].get(x[i]); dv[i].get(d[i]); sv[i].get(s[i]);
      if (!AHEAD) load_gain<1, TPR>(a.gain, lane + i * TPR, a.cols, reinterpret_cast<float(&)[1][8]>(g[i]));
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        x[i][j] *= by;
        dg[i][j] += d[i][j] * x[i][j];
        d[i][j] *= g[i][j];
        c += d[i][j] * x[i][j];
      }
    }
    if (AHEAD && row + step < a.rows) request(row + step);
    c = row_sum<W>(c, red[turn]) * inv;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = lane + i * TPR, n = a.cols - u * 8;
      if (!AHEAD) {
        if (a.d_x && u < upr) sv[i].load((const T*)a.d_x + (size_t)row * a.ld_x + u * 8, n);
        xv[i].get(x[i]); dv[i].get(d[i]); sv[i].get(s[i]);
        load_gain<1, TPR>(a.gain, u, a.cols, reinterpret_cast<float(&)[1][8]>(g[i]));
#pragma unroll
        for (int j = 0; j < 8; ++j) { x[i][j] *= by; d[i][j] *= g[i][j]; }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) s[i][j] += by * (d[i][j] - x[i][j] * c);
      if (u >= upr) continue;
      if (a.d_residual) Unit<T, VEC>::store((T*)a.d_residual + (size_t)row * a.ld_residual + u * 8, s[i], n);
      if (a.d_y) {
        if (a.drop.limit) drop8(s[i], row, u, a.drop);
        Unit<T, VEC>::store((T*)a.d_y + (size_t)row * a.ld_y + u * 8, s[i], n);
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

// d_gain: the partial rows in order, 16 threads a column that take a part of them each (512 rows of 2048 columns: 4.8 us, 8.4 with four)
__global__ __launch_bounds__(1024) void join_gain_kernel(const float* partial, int groups, int cols, float* d_gain) {
  __shared__ float red[1024];
  const int c = blockIdx.x * 64 + threadIdx.x % 64, part = threadIdx.x / 64;
  const int per = (groups + 15) / 16, lo = part * per, hi = min(groups, lo + per);
  float t = 0.f;
  if (c < cols) {
#pragma unroll 16
    for (int r = lo; r < hi; ++r) t += partial[(size_t)r * cols + c];
  }
  red[threadIdx.x] = t;
  __syncthreads();
  if (part || c >= cols) return;
#pragma unroll
  for (int q = 1; q < 16; ++q) t += red[q * 64 + threadIdx.x];
  d_gain[c] = t;
}

template <typename T, int W, int U, bool VEC>
hipError_t forward_run(const JoinArgs& a, hipStream_t s) {
  const int want = W == 1 ? (a.rows + 3) / 4 : a.rows, most = 4096 / (W == 1 ? 4 : W);
  const dim3 grid(want < most ? want : most), block(W == 1 ? 256 : W * 64);
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
  DDG_LAUNCH(join_gain_kernel, dim3((a.cols + 63) / 64), dim3(1024), 0, s, a.partial, groups, a.cols, a.d_gain);
  return hipGetLastError();
}

// Waves a row and units a lane: one unit as long as 16 waves hold the row (8192 x 2048 in bf16: 25.5 us with 4 waves of one unit, 42.5 with one wave of 4,
// 36.9 with 4 waves of 4, a quarter of them idle; 2048 x 4096 with 8-bit output: 15.6 with 8 waves, 24.8 with 4 of two units). 4096 waves: 24.7 us against
// 25.6 with 8192 and 28.0 with 16384.
template <typename T, bool VEC> hipError_t forward_any(const JoinArgs& a, hipStream_t s) {
  const int upr = (a.cols + 7) / 8;
  if (upr <= 64) return forward_run<T, 1, 1, VEC>(a, s);
  if (upr <= 128) return forward_run<T, 2, 1, VEC>(a, s);
  if (upr <= 256) return forward_run<T, 4, 1, VEC>(a, s);
  if (upr <= 512) return forward_run<T, 8, 1, VEC>(a, s);
  if (upr <= 1024) return forward_run<T, 16, 1, VEC>(a, s);
  if (upr <= 2048) return forward_run<T, 16, 2, VEC>(a, s);
  return forward_run<T, 16, 4, VEC>(a, s);
}
template <typename T, bool VEC> hipError_t backward_any(const JoinArgs& a, hipStream_t s) {
  const int upr = (a.cols + 7) / 8;
  if (upr <= 64) return backward_run<T, 1, 1, VEC>(a, s);
  if (upr <= 128) return backward_run<T, 2, 1, VEC>(a, s);
  if (upr <= 256) return backward_run<T, 4, 1, VEC>(a, s);
  if (upr <= 512) return backward_run<T, 8, 1, VEC>(a, s);
  if (upr <= 1024) return backward_run<T, 16, 1, VEC>(a, s);
  if (upr <= 2048) return backward_run<T, 16, 2, VEC>(a, s);
  return backward_run<T, 16, 4, VEC>(a, s);
}

}  // namespace

// Two workgroups of up to 4 waves a compute unit, or one of more: fewer leave the memory idle (8192 x 2048 in bf16: 35.8 us with 256 workgroups of 4 waves, 32.4 with 512,
// 37.2 with 1024), and more mean more rows to add up afterwards
int join_groups(int rows, int cols) {
  const int upr = (cols + 7) / 8, per = upr <= 64 ? 4 : 1;
  const int most = upr <= 256 ? 512 : 256, want = (rows + per - 1) / per;
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
