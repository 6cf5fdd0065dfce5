// Rows of tokens in registers: what the elementwise kernels of token models (joins, rotary positions) share.
#pragma once
#include "ddg_device.h"

namespace ddg {
namespace {

// 16 bytes on their boundary; past the caches where the call's results are more than they hold: then nothing else is driven out for what the next kernel has to fetch from memory anyway
// (8192 rows of 40 heads of 128 in bf16, turned: 26 us instead of 34, and 60 instead of 62 with the next reader; a quarter of the rows: 17.0 against 15.4 with the reader)
constexpr size_t CACHED = 32u << 20;                       // the dies' L2 together
template <typename V> __device__ __forceinline__ void put16(V* to, V v, bool past) {
  if (past) {
    asm volatile("" ::: "memory");                         // (without these the compiler makes one ordinary store of the two)
    __builtin_nontemporal_store(__builtin_bit_cast(u32x4_t, v), reinterpret_cast<u32x4_t*>(to));
    asm volatile("" ::: "memory");
  } else {
    *to = v;
  }
}

// 8 columns of a row, as they lie in memory. VEC: 16-byte pieces on their boundaries. Otherwise pieces wherever they begin (gfx950 loads and stores
// them there too), and the row's last columns, where fewer than 8 are left, one by one with zeros behind them.
template <typename T, bool VEC> struct Unit {
  static constexpr int PIECES = 8 / Store<T>::VEC;
  typedef typename Store<T>::vec_t piece_t;
  piece_t v[PIECES];
  __device__ __forceinline__ void load(const T* p, int n) {
    if (VEC) {
#pragma unroll
      for (int i = 0; i < PIECES; ++i) v[i] = reinterpret_cast<const piece_t*>(p)[i];
    } else if (n >= 8) {
      __builtin_memcpy(v, p, sizeof(v));
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
  __device__ static __forceinline__ void store(T* p, const float (&o)[8], int n, bool past = false) {
    Unit q;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      float t[Store<T>::VEC];
#pragma unroll
      for (int j = 0; j < Store<T>::VEC; ++j) t[j] = o[i * Store<T>::VEC + j];
      Store<T>::store_vec(reinterpret_cast<T*>(&q.v[i]), t);
    }
    if (VEC) {
#pragma unroll
      for (int i = 0; i < PIECES; ++i) put16(reinterpret_cast<piece_t*>(p) + i, q.v[i], past);
    } else if (n >= 8) {
      __builtin_memcpy(p, q.v, sizeof(q.v));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) if (i < n) Store<T>::store1(p + i, o[i]);
    }
  }
};

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

// The gain of a lane's columns, in registers over all the rows that it takes; 1 where there is none
template <int U, int TPR> __device__ __forceinline__ void load_gain(const float* gain, int lane, int cols, float (&g)[U][8]) {
#pragma unroll
  for (int i = 0; i < U; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int c = (lane + i * TPR) * 8 + j;
      g[i][j] = gain && c < cols ? gain[c] : 1.f;
    }
}

// 8 columns of a row from column c on, zeros behind the row's end, without a conditional load (where branches meet, the compiler waits for all loads in flight): what lies past
// the end is read from the row's last 8 columns and moved into place when it is needed.
template <typename T, bool VEC> struct Row8 {
  Unit<T, VEC> v;
  int past;                                                // columns that were read before c; 8: nothing is there
  __device__ __forceinline__ void load(const T* row, int c, int cols) {
    const int from = VEC || cols >= 8 ? min(c, cols - 8) : 0;
    past = min(c - from, 8);
    if (VEC || cols >= 8) {
      v.load(row + from, 8);
    } else {
      T e[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) e[i] = row[min(i, cols - 1)];
      __builtin_memcpy(&v, e, sizeof(e));
      if (c == 0) past = cols - 8;                         // (fewer than 8 columns: those from `cols` on are not there)
    }
  }
  __device__ __forceinline__ void zero() { v.zero(); past = 0; }
  __device__ __forceinline__ void get(float (&o)[8]) const {
    v.get(o);
    if (VEC) {
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] = past ? 0.f : o[i];
    } else {
#pragma unroll
      for (int k = 4; k; k >>= 1)
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = past > 0 && (past & k) ? (i + k < 8 ? o[i + k] : 0.f) : o[i];
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] = past == 8 || (past < 0 && i >= 8 + past) ? 0.f : o[i];
    }
  }
};
// The same of fp32 [cols], `fill` where there is none
__device__ __forceinline__ void columns8(const float* p, int c, int cols, float fill, float (&o)[8]) {
  if (!p) {
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = fill;
    return;
  }
  Row8<float, false> r;                                    // (vectors may lie anywhere)
  r.load(p, c, cols);
  r.get(o);
}

inline bool aligned(const void* p, long ld, size_t size, size_t to) { return !p || ((uintptr_t)p % to == 0 && (size_t)ld * size % to == 0); }

}  // namespace
}  // namespace ddg
