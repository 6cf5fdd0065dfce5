// The end of a block and the start of the next one: the norm after the block (over a row or over each group of its columns), its gate, the residual, and the norm
// before the next block,
//   u = gain_y y rstd_y,   x = residual_scale residual + scale act(gate) u,   out = gain_x x rstd_x,   rstd = (mean of squares + eps)^-1/2.
// With xhat = x rstd_x, yhat = y rstd_y and c = mean(gain_x d_out xhat), backward:
//   t = d_x + rstd_x (gain_x d_out - xhat c),  d_residual = residual_scale t,  d_u = scale act t,  d_gate = scale t u act',
//   d_y = rstd_y (gain_y d_u - yhat mean(gain_y d_u yhat)),  d_gain_y = sum d_u yhat,  d_gain_x = sum d_out xhat.
// Bound by memory: a row is held in registers, every operand is read once and every result written once, rounded once from 32 bits
// (8192 x 2048 in bf16, a norm per 128 columns, silu: 35 us forward, 168 MB, 4.8 TB/s; 63 us backward, 268 MB, 4.2 TB/s).
#include "ddg_mixing.h"
#include "ddg_rows.h"

namespace ddg {
namespace {

// A unit of 8 columns a lane. 16 waves have 128 registers a lane, which leaves none for the next row's operands (4096 x 8192 in bf16, backward: 121 us; 8 waves of two units, whose
// registers do not fit, 177). Backward only aligned bf16 rows without a column gate fit at all: the other seven forms spill 22 to 78 of a row's own (119 us with a column gate, 264 unaligned; fp32 319).
constexpr int U = 1;

// Sum over the `lanes` (a power of two) neighbouring lanes that share a norm, in each of them
__device__ __forceinline__ float lanes_sum(float v, int lanes) {
  if (lanes > 1) v += dpp_move<0xB1>(v);
  if (lanes > 2) v += dpp_move<0x4E>(v);
  if (lanes > 4) v += dpp_move<0x141>(v);
  if (lanes > 8) v += dpp_move<0x140>(v);
  if (lanes > 16) v += __shfl_xor(v, 16);
  if (lanes > 32) v += __shfl_xor(v, 32);
  return v;
}

// The gate's factor and its slope. With e = exp(-|g|) the sigmoid and what it lacks to 1 are 1 / (1 + e) and e / (1 + e), in one order or the other: neither is a difference, so
// both are good where the gate is all but closed or open. Of bf16 rows by the instructions for exp2 and 1 / x (within 2^-23 (2 + |g|)), of fp32 ones to their last bits.
template <typename T> __device__ __forceinline__ float gate_of(int mode, float g, float& slope) {
  if (mode <= GATE_PLAIN) { slope = 1.f; return g; }
  const float e = sizeof(T) == 2 ? __expf(-fabsf(g)) : expf(-fabsf(g));
  const float large = sizeof(T) == 2 ? __builtin_amdgcn_rcpf(1.f + e) : 1.f / (1.f + e), small = e * large;
  const float sig = g < 0.f ? small : large, rest = g < 0.f ? large : small;
  if (mode == GATE_SIGMOID) { slope = sig * rest; return sig; }
  slope = sig * (1.f + g * rest);
  return g * sig;
}

// COLUMN: the gate is a factor of each column, else a tensor or nothing
template <typename T, int W, bool VEC, bool COLUMN>
__global__ __launch_bounds__(W == 1 ? 256 : W * 64) void gated_forward_kernel(GatedArgs a) {
  constexpr int TPR = W * 64, RPB = W == 1 ? 4 : 1;
  constexpr bool AHEAD = W < 16;
  __shared__ float red[2][2][W];
  const int lane = threadIdx.x % TPR, upr = (a.cols + 7) / 8, step = gridDim.x * RPB, lanes = a.group / 8;
  const int shift = a.group ? __builtin_ctz(lanes) : 0;
  const bool wide = !COLUMN && a.mode >= GATE_PLAIN;
  int row = blockIdx.x * RPB + threadIdx.x / TPR;
  Row8<T, VEC> yv[U], rv[U], gv[U];
  auto request = [&](int r) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int c = (lane + i * TPR) * 8;
      yv[i].load((const T*)a.y + (size_t)r * a.ld_y, c, a.cols);
      if (wide) gv[i].load((const T*)a.gate + (size_t)r * a.ld_gate, c, a.cols);
      if (a.residual) rv[i].load((const T*)a.residual + (size_t)r * a.ld_residual, c, a.cols);
    }
  };
#pragma unroll
  for (int i = 0; i < U; ++i) { yv[i].zero(); rv[i].zero(); gv[i].zero(); }
  if (AHEAD && row < a.rows) request(row);
  float gy[U][8], gx[U][8], gc[U][8];
  {
#pragma unroll
    for (int i = 0; i < U; ++i) columns8(a.gain_y, (lane + i * TPR) * 8, a.cols, 1.f, gy[i]);
#pragma unroll
    for (int i = 0; i < U; ++i) columns8(a.gain_x, (lane + i * TPR) * 8, a.cols, 1.f, gx[i]);
#pragma unroll
    for (int i = 0; i < U; ++i) columns8(COLUMN ? (const float*)a.gate : nullptr, (lane + i * TPR) * 8, a.cols, 1.f, gc[i]);
  }
  const float inv = 1.f / (float)a.cols, inv_group = a.group ? 1.f / (float)a.group : inv;
  for (int turn = 0; row < a.rows; row += step, turn ^= 1) {
    if (!AHEAD) request(row);
    float y[U][8], x[U][8], g[U][8], ss = 0.f;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      yv[i].get(y[i]); rv[i].get(x[i]); gv[i].get(g[i]);
#pragma unroll
      for (int j = 0; j < 8; ++j) ss += y[i][j] * y[i][j];
    }
    if (AHEAD && row + step < a.rows) request(row + step);
    float whole = 0.f;
    if (!a.group) whole = rsqrtf(row_sum<W>(ss, red[turn][0]) * inv + a.eps);
    if (!a.group && a.rstd_y && lane == 0) a.rstd_y[row] = whole;
    ss = 0.f;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = lane + i * TPR, n = a.cols - u * 8;
      float rstd = whole;
      if (a.group) {
        float t = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) t += y[i][j] * y[i][j];
        rstd = rsqrtf(lanes_sum(t, lanes) * inv_group + a.eps);
        if (a.rstd_y && u < upr && (u & (lanes - 1)) == 0) a.rstd_y[(size_t)row * (upr >> shift) + (u >> shift)] = rstd;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float slope;
        const float act = wide ? gate_of<T>(a.mode, g[i][j], slope) : gc[i][j];
        x[i][j] = a.residual_scale * x[i][j] + a.scale * (act * (y[i][j] * rstd * gy[i][j]));
        ss += x[i][j] * x[i][j];
      }
      if (a.x && u < upr) Unit<T, VEC>::store((T*)a.x + (size_t)row * a.ld_x + u * 8, x[i], n, a.past);
    }
    if (!a.out && !a.rstd_x) continue;
    const float rstd = rsqrtf(row_sum<W>(ss, red[turn][1]) * inv + a.eps);
    if (a.rstd_x && lane == 0) a.rstd_x[row] = rstd;
    if (!a.out) continue;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = lane + i * TPR, n = a.cols - u * 8;
#pragma unroll
      for (int j = 0; j < 8; ++j) x[i][j] = x[i][j] * rstd * gx[i][j];
      if (u < upr) Unit<T, VEC>::store((T*)a.out + (size_t)row * a.ld_out + u * 8, x[i], n, a.past);
    }
  }
}

// A workgroup's rows of d_gain_y, d_gain_x and a column gate's d_gate stay in registers over all the rows that it takes: one row of `partial` each in the end (rows of whole units: 16-byte
// stores; one by one they took 6 us of 23 with 777 fp32 rows of 1001), no atomics, so the bits do not depend on the order of workgroups.
template <typename T, int W, bool VEC, bool COLUMN>
__global__ __launch_bounds__(W == 1 ? 256 : W * 64) void gated_backward_kernel(GatedArgs a) {
  constexpr int TPR = W * 64, RPB = W == 1 ? 4 : 1;
  constexpr bool AHEAD = W < 16;
  __shared__ float red[2][2][W];
  __shared__ float joined[W == 1 ? 3 : 1][W == 1 ? U * 512 : 1];
  const int lane = threadIdx.x % TPR, part = threadIdx.x / TPR, step = gridDim.x * RPB;
  const int upr = (a.cols + 7) / 8, lanes = a.group / 8, shift = a.group ? __builtin_ctz(lanes) : 0, per_row = a.group ? upr >> shift : 1;
  const bool wide = !COLUMN && a.mode >= GATE_PLAIN;
  Row8<T, VEC> xv[U], yv[U], gv[U], dv[U], sv[U];
  float ry[U], rx = 0.f;
  auto request = [&](int r) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = lane + i * TPR, c = u * 8;
      yv[i].load((const T*)a.y + (size_t)r * a.ld_y, c, a.cols);
      if (wide) gv[i].load((const T*)a.gate + (size_t)r * a.ld_gate, c, a.cols);
      if (a.d_out) {
        xv[i].load((const T*)a.x + (size_t)r * a.ld_x, c, a.cols);
        dv[i].load((const T*)a.d_out + (size_t)r * a.ld_out, c, a.cols);
      }
      if (a.d_x) sv[i].load((const T*)a.d_x + (size_t)r * a.ld_x, c, a.cols);
      ry[i] = a.rstd_y[(size_t)r * per_row + (a.group ? min(u >> shift, per_row - 1) : 0)];
    }
    if (a.d_out) rx = a.rstd_x[r];
  };
  float dgy[U][8], dgx[U][8], dgc[U][8], gy[U][8], gx[U][8], gc[U][8];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    xv[i].zero(); yv[i].zero(); gv[i].zero(); dv[i].zero(); sv[i].zero(); ry[i] = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) dgy[i][j] = dgx[i][j] = dgc[i][j] = 0.f;
  }
  int row = blockIdx.x * RPB + part;
  if (AHEAD && row < a.rows) request(row);
  {
#pragma unroll
    for (int i = 0; i < U; ++i) columns8(a.gain_y, (lane + i * TPR) * 8, a.cols, 1.f, gy[i]);
#pragma unroll
    for (int i = 0; i < U; ++i) columns8(a.gain_x, (lane + i * TPR) * 8, a.cols, 1.f, gx[i]);
#pragma unroll
    for (int i = 0; i < U; ++i) columns8(COLUMN ? (const float*)a.gate : nullptr, (lane + i * TPR) * 8, a.cols, 1.f, gc[i]);
  }
  const float inv = 1.f / (float)a.cols, inv_group = a.group ? 1.f / (float)a.group : inv;
  for (int turn = 0; row < a.rows; row += step, turn ^= 1) {
    if (!AHEAD) request(row);
    float x[U][8], d[U][8], y[U][8], g[U][8], s[U][8], by[U], c = 0.f;
    const float rstd = rx;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = lane + i * TPR;
      xv[i].get(x[i]); dv[i].get(d[i]); yv[i].get(y[i]); gv[i].get(g[i]); sv[i].get(s[i]);
      by[i] = ry[i];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        x[i][j] *= rstd;
        dgx[i][j] += d[i][j] * x[i][j];
        d[i][j] *= gx[i][j];
        c += d[i][j] * x[i][j];
      }
    }
    if (AHEAD && row + step < a.rows) request(row + step);
    if (a.d_out) c = row_sum<W>(c, red[turn][0]) * inv;
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = lane + i * TPR, n = a.cols - u * 8;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float slope = 1.f;
        const float act = wide ? gate_of<T>(a.mode, g[i][j], slope) : gc[i][j];
        const float t = s[i][j] + rstd * (d[i][j] - x[i][j] * c), scaled = a.scale * t;
        s[i][j] = a.residual_scale * t;
        y[i][j] *= by[i];                                     // yhat
        g[i][j] = scaled * (y[i][j] * gy[i][j]) * slope;      // d_gate
        if (COLUMN) dgc[i][j] += g[i][j];
        d[i][j] = scaled * act;                               // d_u
        dgy[i][j] += d[i][j] * y[i][j];
        d[i][j] *= gy[i][j];
        m += d[i][j] * y[i][j];
      }
      if (u < upr && a.d_residual) Unit<T, VEC>::store((T*)a.d_residual + (size_t)row * a.ld_residual + u * 8, s[i], n, a.past);
      if (u < upr && wide && a.d_gate) Unit<T, VEC>::store((T*)a.d_gate + (size_t)row * a.ld_gate + u * 8, g[i], n, a.past);
      if (a.group && a.d_y) {
        m = lanes_sum(m, lanes) * inv_group;
#pragma unroll
        for (int j = 0; j < 8; ++j) s[i][j] = by[i] * (d[i][j] - y[i][j] * m);
        if (u < upr) Unit<T, VEC>::store((T*)a.d_y + (size_t)row * a.ld_y + u * 8, s[i], n, a.past);
        m = 0.f;
      }
    }
    if (a.group || !a.d_y) continue;
    m = row_sum<W>(m, red[turn][1]) * inv;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = lane + i * TPR, n = a.cols - u * 8;
#pragma unroll
      for (int j = 0; j < 8; ++j) s[i][j] = by[i] * (d[i][j] - y[i][j] * m);
      if (u < upr) Unit<T, VEC>::store((T*)a.d_y + (size_t)row * a.ld_y + u * 8, s[i], n, a.past);
    }
  }
  auto leave = [&](float (&v)[U][8], int which) __attribute__((always_inline)) {
    if (W == 1) {
      __syncthreads();
      if (part) {
#pragma unroll
        for (int i = 0; i < U; ++i)
#pragma unroll
          for (int j = 0; j < 8; ++j) joined[part - 1][(i * 8 + j) * 64 + lane] = v[i][j];
      }
      __syncthreads();
      if (part) return;
#pragma unroll
      for (int i = 0; i < U; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int q = 0; q < 3; ++q) v[i][j] += joined[q][(i * 8 + j) * 64 + lane];
    }
    float* to = a.partial + ((size_t)which * gridDim.x + blockIdx.x) * (upr * 8);
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = lane + i * TPR;
      if (u >= upr) continue;
      Store<float>::store4(to + u * 8, v[i][0], v[i][1], v[i][2], v[i][3]);
      Store<float>::store4(to + u * 8 + 4, v[i][4], v[i][5], v[i][6], v[i][7]);
    }
  };
  if (a.d_gain_y) leave(dgy, 0);
  if (a.d_gain_x) leave(dgx, 1);
  if (COLUMN && a.d_gate) leave(dgc, 2);
}

// The partial rows in order, 16 threads a column that take a part of them each; a row of workgroups for each of the sums
__global__ __launch_bounds__(1024) void gated_gain_kernel(const float* partial, int groups, int cols, float* d_gain_y, float* d_gain_x, float* d_gate) {
  float* const to = blockIdx.y == 0 ? d_gain_y : blockIdx.y == 1 ? d_gain_x : d_gate;
  if (!to) return;
  const int ld = (cols + 7) / 8 * 8;
  partial += (size_t)blockIdx.y * groups * ld;
  __shared__ float red[1024];
  const int c = blockIdx.x * 64 + threadIdx.x % 64, part = threadIdx.x / 64;
  const int per = (groups + 15) / 16, lo = part * per, hi = min(groups, lo + per);
  float t = 0.f;
  if (c < cols) {
#pragma unroll 16
    for (int r = lo; r < hi; ++r) t += partial[(size_t)r * ld + c];
  }
  red[threadIdx.x] = t;
  __syncthreads();
  if (part || c >= cols) return;
#pragma unroll
  for (int q = 1; q < 16; ++q) t += red[q * 64 + threadIdx.x];
  to[c] = t;
}

template <typename T, int W, bool VEC> hipError_t forward_run(const GatedArgs& a, hipStream_t s) {
  const int want = W == 1 ? (a.rows + 3) / 4 : a.rows, most = 4096 / (W == 1 ? 4 : W);
  const dim3 grid(want < most ? want : most), block(W == 1 ? 256 : W * 64);
  if (a.mode == GATE_COLUMN) DDG_LAUNCH((gated_forward_kernel<T, W, VEC, true>), grid, block, 0, s, a);
  else DDG_LAUNCH((gated_forward_kernel<T, W, VEC, false>), grid, block, 0, s, a);
  return hipGetLastError();
}
template <typename T, int W, bool VEC> hipError_t backward_run(const GatedArgs& a, hipStream_t s) {
  const int groups = gated_groups(a.rows, a.cols);
  const dim3 block(W == 1 ? 256 : W * 64);
  if (a.mode == GATE_COLUMN) DDG_LAUNCH((gated_backward_kernel<T, W, VEC, true>), dim3(groups), block, 0, s, a);
  else DDG_LAUNCH((gated_backward_kernel<T, W, VEC, false>), dim3(groups), block, 0, s, a);
  const hipError_t e = hipGetLastError();
  float* d_gate = a.mode == GATE_COLUMN ? (float*)a.d_gate : nullptr;
  if (e != hipSuccess || !(a.d_gain_y || a.d_gain_x || d_gate)) return e;
  DDG_LAUNCH(gated_gain_kernel, dim3((a.cols + 63) / 64, d_gate ? 3 : 2), dim3(1024), 0, s, a.partial, groups, a.cols, a.d_gain_y, a.d_gain_x, d_gate);
  return hipGetLastError();
}

template <typename T, bool VEC> hipError_t forward_any(const GatedArgs& a, hipStream_t s) {
  const int upr = (a.cols + 7) / 8;
  if (upr <= 64) return forward_run<T, 1, VEC>(a, s);
  if (upr <= 128) return forward_run<T, 2, VEC>(a, s);
  if (upr <= 256) return forward_run<T, 4, VEC>(a, s);
  if (upr <= 512) return forward_run<T, 8, VEC>(a, s);
  return forward_run<T, 16, VEC>(a, s);
}
template <typename T, bool VEC> hipError_t backward_any(const GatedArgs& a, hipStream_t s) {
  const int upr = (a.cols + 7) / 8;
  if (upr <= 64) return backward_run<T, 1, VEC>(a, s);
  if (upr <= 128) return backward_run<T, 2, VEC>(a, s);
  if (upr <= 256) return backward_run<T, 4, VEC>(a, s);
  if (upr <= 512) return backward_run<T, 8, VEC>(a, s);
  return backward_run<T, 16, VEC>(a, s);
}

}  // namespace

int gated_groups(int rows, int cols) {
  const int upr = (cols + 7) / 8, per = upr <= 64 ? 4 : 1;
  const int most = upr <= 256 ? 512 : 256, want = (rows + per - 1) / per;
  return want < 1 ? 1 : want < most ? want : most;
}

hipError_t gated_forward_launch(const GatedArgs& given, hipStream_t s) {
  GatedArgs a = given;
  const size_t size = dtype_size(a.dtype);
  a.past = (size_t)a.rows * a.cols * size * ((a.x != nullptr) + (a.out != nullptr)) > CACHED;
  const bool vec = a.cols % 8 == 0 && aligned(a.y, a.ld_y, size, 16) && (a.mode < GATE_PLAIN || aligned(a.gate, a.ld_gate, size, 16)) &&
                   aligned(a.residual, a.ld_residual, size, 16) && aligned(a.x, a.ld_x, size, 16) && aligned(a.out, a.ld_out, size, 16);
  if (a.dtype == BF16) return vec ? forward_any<bf16_t, true>(a, s) : forward_any<bf16_t, false>(a, s);
  return vec ? forward_any<float, true>(a, s) : forward_any<float, false>(a, s);
}

hipError_t gated_backward_launch(const GatedArgs& given, hipStream_t s) {
  GatedArgs a = given;
  const size_t size = dtype_size(a.dtype);
  a.past = (size_t)a.rows * a.cols * size * ((a.d_residual != nullptr) + (a.d_y != nullptr) + (a.mode >= GATE_PLAIN && a.d_gate)) > CACHED;
  const bool vec = a.cols % 8 == 0 && aligned(a.y, a.ld_y, size, 16) && aligned(a.d_y, a.ld_y, size, 16) && aligned(a.x, a.ld_x, size, 16) &&
                   (a.mode < GATE_PLAIN || (aligned(a.gate, a.ld_gate, size, 16) && aligned(a.d_gate, a.ld_gate, size, 16))) &&
                   aligned(a.d_x, a.ld_x, size, 16) && aligned(a.d_out, a.ld_out, size, 16) && aligned(a.d_residual, a.ld_residual, size, 16);
  if (a.dtype == BF16) return vec ? backward_any<bf16_t, true>(a, s) : backward_any<bf16_t, false>(a, s);
  return vec ? backward_any<float, true>(a, s) : backward_any<float, false>(a, s);
}

}  // namespace ddg
