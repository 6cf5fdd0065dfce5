// Linear attention with a decay g = exp(log_decay) for each head, in chunks of 64 rows. With S_t = sum_{s<=t} g^(t-s) k_s v_s^T the definition is
//   o_t = scale S_t^T q_t.  Backward: dq_t = scale S_t do_t,  dk_t = R_t v_t,  dv_t = R_t^T k_t,  R_t = scale sum_{s>=t} g^(s-t) q_s do_s^T (+ the gradient of the last state).
// All four are one walk over a sequence, forwards or from its end (LinearJob): a chunk of rows x, a, b with the state S before it (K x V) gives
//   out_r = inter g^(r+1-late) x_r S + intra sum_{j<=r} g^(r-j) (x_r . a_j) b_j,    S <- g^n S + update sum_j g^(n-1-j+late) a_j b_j^T:
// three matrix products of 64 rows for each of S's 64-column slices, 4 K V flops a row in the end where the sum over all pairs would take T (K + V).
// A workgroup of four waves walks over a sequence (or a segment of one) for one head and one slice; S stays in its registers in 32 bits and goes to LDS once a chunk,
// as the operand of the next product. One prompt of 16384 rows, 16 heads of 128, bf16: 135 us, of which the walk 90 (276 MB, 3.1 TB/s; vector, matrix and LDS
// instructions take a third of its cycles each and overlap little), gradients of 8 sequences of 1024 rows 118 us. Where there are fewer sequences and heads than the chip holds, sequences are cut into segments: a pass that only adds up
// each segment's own state, a short scan over the segments, and the walk, which starts each segment from the state that the scan left.
#include "ddg_mixing.h"
#include "ddg_rows.h"

#include <type_traits>

namespace ddg {
namespace {

constexpr int CHUNK = 64, SLICE = 64;

typedef short tr4_t __attribute__((ext_vector_type(4)));
typedef unsigned u32x2_t __attribute__((ext_vector_type(2)));
typedef tr4_t __attribute__((address_space(3))) * tr_ptr_t;

// What the two types do differently. A fragment holds KV consecutive values of the contracted index for one row or column (Mma in ddg_device.h).
// across(): of a tile [rows][columns] in LDS the fragment whose contracted index runs over rows: those of the 16-row tiles that an accumulator has in the same lane,
// 16 t + 4 (lane / 16) .. + 3, for as many tiles t as it takes (bf16: two). So products P that lie in accumulators are fragments without an exchange.
template <typename T> struct Mix;
template <> struct Mix<bf16_t> {
  typedef Mma<bf16_t> M;
  static constexpr int PAD = 16, TILES = 2, PLANES = 2;
  // in every block of 16 lanes, lane s gives the address of 4 columns of row s / 4 and gets column s of the four rows
  __device__ static __forceinline__ M::frag_t across(const bf16_t* tile, int ld, int step, int col, int lane) {
    const bf16_t* p = tile + (32 * step + 4 * (lane >> 4) + ((lane & 15) >> 2)) * ld + col + 4 * (lane & 3);
    const uint2 l = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr_t)(p)));
    const uint2 h = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr_t)(p + 16 * ld)));
    return make_uint4(l.x, l.y, h.x, h.y);
  }
  // an accumulator's values as operands, the sum of two: 16 bits, so that the result is rounded once
  __device__ static __forceinline__ void split(const f32x4_t& p, uint2& h, uint2& l) {
    h = make_uint2(f32x2_to_bf16x2(p[0], p[1]), f32x2_to_bf16x2(p[2], p[3]));
    l = make_uint2(f32x2_to_bf16x2(p[0] - __uint_as_float(h.x << 16), p[1] - __uint_as_float(h.x & 0xffff0000u)),
                   f32x2_to_bf16x2(p[2] - __uint_as_float(h.y << 16), p[3] - __uint_as_float(h.y & 0xffff0000u)));
  }
  __device__ static __forceinline__ void pack(const f32x4_t* p, M::frag_t (&o)[2]) {
    uint2 h[2], l[2];
    split(p[0], h[0], l[0]);
    split(p[1], h[1], l[1]);
    o[0] = make_uint4(h[0].x, h[0].y, h[1].x, h[1].y);
    o[1] = make_uint4(l[0].x, l[0].y, l[1].x, l[1].y);
  }
};
template <> struct Mix<float> {
  typedef Mma<float> M;
  static constexpr int PAD = 4, TILES = 1, PLANES = 1;
  __device__ static __forceinline__ M::frag_t across(const float* tile, int ld, int step, int col, int lane) {
    const float* p = tile + (16 * step + 4 * (lane >> 4)) * ld + col + (lane & 15);
    return make_float4(p[0], p[ld], p[2 * ld], p[3 * ld]);
  }
  __device__ static __forceinline__ void pack(const f32x4_t* p, M::frag_t (&o)[1]) { o[0] = make_float4(p[0][0], p[0][1], p[0][2], p[0][3]); }
};

// The state as an operand in LDS: 64 rows (its columns) of DK values. Piece p of row r lies at p ^ place: readers take a piece of 16 rows at once, and writers half a piece of 16 rows,
// which padded rows would send to a quarter of the banks (a third of all LDS cycles).
template <typename T, int DK> struct State {
  static constexpr int PIECES = DK * (int)sizeof(T) / 16, W = 16 / (int)sizeof(T);
  static constexpr int PLACES = PIECES % 16 == 0 ? 16 : PIECES % 8 == 0 ? 8 : 4, ROWS = PIECES < 16 && PIECES % 12 ? 16 / PIECES : 1;     // (rows in 256 bytes)
  __device__ static __forceinline__ int at(int r, int p) { return r * DK + (p ^ (r / ROWS & (PLACES - 1))) * W; }
};

// Whether any of a piece's elements is infinite or NaN: all bits of its exponent are set
__device__ __forceinline__ bool beyond(uint4 v) {
  const auto carry = [](unsigned u) { return (u & 0x7f807f80u) + 0x00800080u; };     // (bf16 pairs: a set exponent's carry ends in the sign's place)
  return ((carry(v.x) | carry(v.y) | carry(v.z) | carry(v.w)) & 0x80008000u) != 0;
}
__device__ __forceinline__ bool beyond(float4 v) { return !(fabsf(v.x) < INFINITY && fabsf(v.y) < INFINITY && fabsf(v.z) < INFINITY && fabsf(v.w) < INFINITY); }

// b times the rows' weights, as N fragments whose sum it is: bf16 keeps 8 bits of the product in each, fp32 all of them
template <int N> __device__ __forceinline__ void weigh(uint4 b, const float* w, uint4 (&o)[N]) {
  float v[8];
  Store<bf16_t>::unpack_vec(b, v);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] *= w[i];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    o[k] = make_uint4(f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3]), f32x2_to_bf16x2(v[4], v[5]), f32x2_to_bf16x2(v[6], v[7]));
    if (k + 1 == N) break;
    float u[8];
    Store<bf16_t>::unpack_vec(o[k], u);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] -= u[i];
  }
}
template <int N> __device__ __forceinline__ void weigh(float4 b, const float* w, float4 (&o)[N]) {
  o[0] = make_float4(b.x * w[0], b.y * w[1], b.z * w[2], b.w * w[3]);
}

// The rows of a chunk of one operand, and 16 bytes of a row, zeros where there is nothing: no load is conditional, since where branches meet the compiler waits for
// all loads in flight. VEC: whole 16-byte pieces through a resource, what lies outside at NOWHERE. Otherwise pieces wherever they begin, from the nearest place that
// has them (the first row, the end of the row), put right by settle() when they are needed.
template <typename T, bool VEC> struct Rows;
template <typename T> struct Rows<T, true> {
  typedef typename Mma<T>::frag_t frag_t;
  wide_rsrc_t res;
  unsigned step, top;
  int n, cols;
  // row r of the chunk is at p + r * stride; n rows of `cols` columns
  __device__ __forceinline__ void at(const T* p, long stride, int n_, int cols_) {
    over(p, 0, stride, sizeof(T));
    n = n_; cols = cols_;
  }
  // the same at element `from` of p, of elements of `size` bytes; p null: nowhere
  __device__ __forceinline__ void over(const void* p, long from, long stride, int size) {
    const bool back = stride < 0;
    const uint64_t q = (uint64_t)(uintptr_t)p + (uint64_t)((back ? from + (CHUNK - 1) * stride : from) * size);
    const uint64_t u = (uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)q) | (uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)(q >> 32)) << 32;
    res = wide_rsrc((const void*)(uintptr_t)u, p ? 0x80000000u : 0u);
    const unsigned by = (unsigned)((back ? -stride : stride) * size);
    step = back ? 0u - by : by;
    top = back ? (CHUNK - 1) * by : 0u;
  }
  __device__ __forceinline__ frag_t get(int r, int c) const {
    return __builtin_bit_cast(frag_t, wide_load(res, r < n && c < cols ? top + (unsigned)r * step + (unsigned)c * (unsigned)sizeof(T) : NOWHERE, 0));
  }
  __device__ __forceinline__ frag_t settle(frag_t v, int, int) const { return v; }
};
template <typename T> struct Rows<T, false> {
  typedef typename Mma<T>::frag_t frag_t;
  static constexpr int W = Mma<T>::KV;
  const T* p;
  long stride;
  int n, cols;
  __device__ __forceinline__ void at(const T* p_, long stride_, int n_, int cols_) { p = p_; stride = stride_; n = n_; cols = cols_; }
  __device__ __forceinline__ frag_t get(int r, int c) const {
    const T* row = p + (r < n ? r : 0) * stride;
    frag_t v;
    if (cols >= W) {
      __builtin_memcpy(&v, row + (c + W <= cols ? c : cols - W), sizeof(v));
    } else {
      T e[W];
#pragma unroll
      for (int i = 0; i < W; ++i) e[i] = row[i < cols ? i : 0];
      __builtin_memcpy(&v, e, sizeof(v));
    }
    return v;
  }
  __device__ __forceinline__ frag_t settle(frag_t f, int r, int c) const {
    const uint4 v = __builtin_bit_cast(uint4, f);
    uint64_t lo = v.x | (uint64_t)v.y << 32, hi = v.z | (uint64_t)v.w << 32;
    if (r >= n || c >= cols) lo = hi = 0;
    if (cols >= W) {                                       // what was read began `past` elements before c
      const int past = c + W <= cols ? 0 : c - (cols - W), bits = (past * (int)sizeof(T) & 7) * 8;
      if (past * (int)sizeof(T) >= 8) { lo = hi; hi = 0; }
      lo = lo >> bits | (bits ? hi << (64 - bits) : 0);
      hi >>= bits;
    } else {
      const int bits = cols * (int)sizeof(T) * 8;          // c is 0
      hi = bits > 64 ? hi & ((1ull << (bits - 64)) - 1) : 0;
      if (bits < 64) lo &= (1ull << bits) - 1;
    }
    return __builtin_bit_cast(frag_t, make_uint4((unsigned)lo, (unsigned)(lo >> 32), (unsigned)hi, (unsigned)(hi >> 32)));
  }
};

// What LDS holds is there for all waves; loads and stores of memory go on
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Where a workgroup is: its sequence, and the rows [first, first + rows) of it, counted in the direction of the walk
struct Place { int sequence, start, length, first, rows, segments, piece; bool none; };

__device__ __forceinline__ int clamp_row(int v, int rows) { return v < 0 ? 0 : v > rows ? rows : v; }
// Segments are numbered so that nobody has to add up lengths: sequence n's are start / segment + n and on, at least one each, and the numbers between are nobody's.
// starts is device data that the host has not seen: everything is held inside [0, rows]. Pieces (states before the segments) have numbers of their own where by_rows says so.
__device__ __forceinline__ Place find(const LinearArgs& g, int number) {
  Place p;
  if (!g.starts) {
    const int length = g.rows / g.sequences, per = g.split ? (length + g.segment - 1) / g.segment : 1, each = per > 0 ? per : 1;
    p.sequence = number / each;
    p.start = p.sequence * length;
    p.length = length;
    p.first = (number - p.sequence * each) * g.segment;
    p.segments = each;
    p.piece = number;
    p.none = p.sequence >= g.sequences;
  } else if (!g.split) {
    p.sequence = number;
    p.start = clamp_row(g.starts[number], g.rows);
    p.length = max(0, clamp_row(g.starts[number + 1], g.rows) - p.start);
    p.first = 0;
    p.segments = 1;
    p.piece = number;
    p.none = false;
  } else {
    // the last sequence whose first number is this one or less; every wave looks for itself, at 64 of them in a trip (they rise; where starts fall, the range still shrinks). 65536 sequences of
    // two rows, 2 heads of 64: 2.1 ms, 25 where every workgroup reads all starts; 4096, 8 heads: 0.51 ms, 0.82
    int n = 0, end = 0;
    p.start = 0;
    p.none = false;
    for (int span = g.sequences, step; ; span = step) {
      step = (span + 63) / 64;
      const int lane = threadIdx.x & 63, of = (int)min((long)n + (long)lane * step, (long)g.sequences - 1);
      const int s0 = clamp_row(g.starts[of], g.rows), s1 = step == 1 ? clamp_row(g.starts[of + 1], g.rows) : 0;
      const int here = __popcll(__ballot(lane * step < span && n + lane * step < g.sequences && s0 / g.segment + of <= number));
      if (here == 0) { p.none = true; break; }
      n += (here - 1) * step;
      if (step == 1) {
        p.start = __shfl(s0, here - 1);
        end = __shfl(s1, here - 1);
        break;
      }
    }
    p.sequence = n;
    p.length = max(0, end - p.start);
    p.first = (int)min((long)(number - (p.start / g.segment + n)) * g.segment, (long)g.rows);
    p.segments = max(1, (p.length + g.segment - 1) / g.segment);
    p.piece = g.by_rows ? 2 * p.start / g.segment + p.first / g.segment : number;
    p.none |= p.first < 0 || (p.first > 0 && p.first >= p.length);     // (starts that fall are found anywhere)
  }
  p.sequence = __builtin_amdgcn_readfirstlane(p.sequence);
  p.start = __builtin_amdgcn_readfirstlane(p.start);
  p.length = __builtin_amdgcn_readfirstlane(p.length);
  p.first = __builtin_amdgcn_readfirstlane(p.first);
  p.segments = __builtin_amdgcn_readfirstlane(p.segments);
  p.piece = __builtin_amdgcn_readfirstlane(p.piece);
  p.rows = p.length - p.first;
  if (g.split && p.rows > g.segment) p.rows = g.segment;
  return p;
}

// Neighbouring numbers on one of the 8 dies, whose L2 then holds what they share: workgroups go to the dies in turn
__device__ __forceinline__ int on_die(int id, int total) {
  const int q = total / 8, r = total % 8, die = id & 7, i = id >> 3;
  return die < r ? die * (q + 1) + i : r * (q + 1) + (die - r) * q + i;
}

// SUM: only the state of the segment's own rows, for the scan. PLANES: fragments a weighted b is taken apart into.
template <typename T, int DK, int PLANES, bool VEC, bool SUM>
__device__ __forceinline__ void walk(const LinearArgs& g) {
  typedef Mma<T> M;
  typedef Mix<T> X;
  typedef typename M::frag_t frag_t;
  typedef State<T, DK> SL;
  constexpr int W = M::KV, LDA = DK + X::PAD, LDB = SLICE + X::PAD, STEPS = DK / M::KSTEP, OVER = 4 / X::TILES, GROUP = DK % 64 ? 2 : 4;
  constexpr int PA = CHUNK * DK / W / 256, PB = CHUNK * SLICE / W / 256;
  extern __shared__ __align__(16) unsigned char smem[];
  T* const at = reinterpret_cast<T*>(smem);                // [64][LDA]
  T* const bt = at + CHUNK * LDA;                          // [64][LDB]
  T* const st = bt + CHUNK * LDB;                          // [PLANES][State]
  __shared__ float pair_power[2 * CHUNK], row_power[2 * CHUNK];
  __shared__ int beyond_at[2];

  const LinearJob job = g.job[blockIdx.y];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, l4 = lane >> 4;
  const int total = g.segments * g.heads * job.slices;
  if ((int)blockIdx.x >= total) return;
  const int number = on_die(blockIdx.x, total), slice = number % job.slices, head = number / job.slices % g.heads;
  const Place place = find(g, number / job.slices / g.heads);
  if constexpr (!VEC && !SUM && sizeof(T) == 2) asm volatile("" ::: "memory");     // (else the compiler moves loads into the search, and unaligned rows of 128 columns spill 25 registers instead of 6)
  if (place.none || (SUM && place.segments == 1)) return;
  const int K = job.K, V = job.V, v0 = slice * SLICE;

  // the rows of the walk: row r of the sequence is at base + r * step
  const long sx = job.back ? -job.ld_x : job.ld_x, sa = job.back ? -job.ld_a : job.ld_a, sb = job.back ? -job.ld_b : job.ld_b;
  const size_t origin = (size_t)place.start + (job.back ? (place.length ? place.length - 1 : 0) : 0);
  const T* const bx = (const T*)job.x + origin * job.ld_x + (size_t)(head / job.share_x) * K + place.first * sx;
  const T* const ba = (const T*)job.a + origin * job.ld_a + (size_t)(head / job.share_a) * K + place.first * sa;
  const T* const bb = (const T*)job.b + origin * job.ld_b + (size_t)(head / job.share_b) * V + place.first * sb + v0;
  const long out_step = job.back ? -job.ld_out : job.ld_out, out_at = (long)origin * job.ld_out + (long)head * V + place.first * out_step;
  const int out_size = job.out_f32 ? 4 : (int)sizeof(T), tile = (blockIdx.x >> 8 & 1) ? 3 - wave : wave, row = 16 * tile + l16;

  frag_t x[STEPS], ar[PA], br[PB];
  Rows<T, VEC> rx, ra, rb;
  auto request = [&](int r0) __attribute__((always_inline)) {
    const int n = min(CHUNK, place.rows - r0);
    ra.at(ba + r0 * sa, sa, n, K);
#pragma unroll
    for (int i = 0; i < PA; ++i) ar[i] = ra.get((tid + i * 256) / (DK / W), (tid + i * 256) % (DK / W) * W);
    rb.at(bb + r0 * sb, sb, n, V - v0);
#pragma unroll
    for (int i = 0; i < PB; ++i) br[i] = rb.get((tid + i * 256) / (SLICE / W), (tid + i * 256) % (SLICE / W) * W);
  };

  // a wave's own rows are free for the next ones before the chunk ends
  auto request_x = [&](int r0) __attribute__((always_inline)) {
    rx.at(bx + r0 * sx, sx, min(CHUNK, place.rows - r0), K);
#pragma unroll
    for (int s = 0; s < STEPS; ++s) x[s] = rx.get(row, s * M::KSTEP + l4 * W);
  };
  if (place.rows > 0) {
    request(0);
    if (!SUM) request_x(0);
  }

  // factors that every chunk shares, 0 from 64 on: intra g^(r-j) at 63 - r + j, update g^(n-1-j+late) at 64 - n + j, inter g^(r+1-late)
  const float lam = g.log_decay[head];
  const auto power = [&](int n) __attribute__((always_inline)) { return n ? expf((float)n * lam) : 1.f; };
  if (tid < 2 * CHUNK) {
    const int n = CHUNK - 1 - tid;
    pair_power[tid] = n < 0 ? 0.f : job.intra * power(n);
    row_power[tid] = n < 0 ? 0.f : job.update * power(n + job.late);
  }
  const float into = job.inter * power(row + 1 - job.late), keep_whole = power(CHUNK);

  // S: this wave's 16 columns, all K rows
  f32x4_t S[DK / 16];
  const int col = v0 + 16 * wave + l16;
  int slot = g.slots ? g.slots[place.sequence] : place.sequence;
  if ((unsigned)slot >= (unsigned)g.pool) slot = -1;
  {
    const float* from = nullptr;
    long rk = job.at_k, rv = job.at_v;
    if (!SUM && place.segments > 1) {
      from = job.pieces + ((size_t)place.piece * g.heads + head) * K * V;
      rk = V; rv = 1;
    } else if (!SUM && job.state_in && slot >= 0) {
      from = job.state_in + ((size_t)slot * g.heads + head) * K * V;
    }
    if (from) {
      from += (col < V ? col : V - 1) * rv;
#pragma unroll
      for (int t = 0; t < DK / 16; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = 16 * t + 4 * l4 + e;
          S[t][e] = from[(r < K ? r : K - 1) * rk];
        }
    }
#pragma unroll
    for (int t = 0; t < DK / 16; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) S[t][e] = from && 16 * t + 4 * l4 + e < K && col < V ? S[t][e] : 0.f;
  }
  __syncthreads();
  float pairs[4][4], weight[16];
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) pairs[t][e] = pair_power[CHUNK - 1 - row + 4 * l4 + 16 * t + e];
  const auto weigh_rows = [&](int n) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) weight[4 * t + e] = row_power[CHUNK - n + 4 * l4 + 16 * t + e];
  };
  weigh_rows(CHUNK);

  if (tid < 2) beyond_at[tid] = 0;
  for (int r0 = 0; r0 < place.rows; r0 += CHUNK) {
    const int n = min(CHUNK, place.rows - r0), turn = r0 / CHUNK & 1;
    lds_barrier();
#pragma unroll
    for (int i = 0; i < PA; ++i) {
      const int p = tid + i * 256, r = p / (DK / W), c = p % (DK / W) * W;
      *reinterpret_cast<frag_t*>(at + r * LDA + c) = ra.settle(ar[i], r, c);
    }
#pragma unroll
    for (int i = 0; i < PB; ++i) {
      const int p = tid + i * 256, r = p / (SLICE / W), c = p % (SLICE / W) * W;
      br[i] = rb.settle(br[i], r, c);
      *reinterpret_cast<frag_t*>(bt + r * LDB + c) = br[i];
    }
    if (!SUM) {
      bool any = false;
#pragma unroll
      for (int i = 0; i < PB; ++i) any |= beyond(br[i]);
      if (any) beyond_at[turn] = 1;
    }
    if (!SUM) {
#pragma unroll
      for (int t = 0; t < DK / 16; ++t) {
        if constexpr (sizeof(T) == 2) {
          T* const to = st + SL::at(16 * wave + l16, 2 * t + (l4 >> 1)) + 4 * (l4 & 1);
          uint2 h, l;
          X::split(S[t], h, l);
          *reinterpret_cast<uint2*>(to) = h;
          *reinterpret_cast<uint2*>(to + SLICE * DK) = l;
        } else {
          Store<float>::store4(reinterpret_cast<float*>(st) + SL::at(16 * wave + l16, 4 * t + l4), S[t][0], S[t][1], S[t][2], S[t][3]);
        }
      }
    }
    lds_barrier();
    if (!SUM) {
#pragma unroll
      for (int s = 0; s < STEPS; ++s) x[s] = rx.settle(x[s], row, s * M::KSTEP + l4 * W);
    }
    if (r0 + CHUNK < place.rows) request(r0 + CHUNK);
    const int special = SUM ? 0 : beyond_at[turn];
    if (!SUM && tid == 0) beyond_at[turn ^ 1] = 0;
    // the state after these rows (before their results, which do not wait for it)
    if (n < CHUNK) weigh_rows(n);
    const float keep = n == CHUNK ? keep_whole : power(n);
#pragma unroll
    for (int t = 0; t < DK / 16; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) S[t][e] *= keep;
#pragma unroll
    for (int s = 0; s < OVER; ++s) {
      frag_t w[PLANES];
      weigh<PLANES>(X::across(bt, LDB, s, 16 * wave, lane), weight + 4 * X::TILES * s, w);
#pragma unroll
      for (int t = 0; t < DK / 16; t += GROUP) {
        frag_t a[GROUP];
#pragma unroll
        for (int i = 0; i < GROUP; ++i) a[i] = X::across(at, LDA, s, 16 * (t + i), lane);
#pragma unroll
        for (int p = 0; p < PLANES; ++p)
#pragma unroll
          for (int i = 0; i < GROUP; ++i) S[t + i] = M::mma(a[i], w[p], S[t + i]);
      }
    }
    if (!SUM) {
      // columns of the result, 16 at a time and four at once, so that no product waits for the one before: from the state
      f32x4_t o[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) o[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < STEPS; ++s)
#pragma unroll
        for (int i = 0; i < 4 * X::PLANES; ++i) o[i & 3] = M::mma(M::load(st + SL::at(16 * i + l16, s * (M::KSTEP / W) + l4)), x[s], o[i & 3]);
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[t][e] *= into;
      // and from the pairs of rows: this wave's 16 rows as columns, theirs and the 16-row tiles before as rows
      const auto mix = [&](auto tiles) __attribute__((always_inline)) {
        constexpr int NT = decltype(tiles)::value, USED = (NT + X::TILES - 1) / X::TILES;
        f32x4_t P[USED * X::TILES];
#pragma unroll
        for (int t = 0; t < USED * X::TILES; ++t) P[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
          for (int t = 0; t < NT; ++t) P[t] = M::mma(M::load(at + (16 * t + l16) * LDA + s * M::KSTEP + l4 * W), x[s], P[t]);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) P[t][e] = t + 1 < NT || 4 * l4 + e <= l16 ? P[t][e] * pairs[t][e] : 0.f;      // (later rows may hold anything)
#pragma unroll
        for (int s = 0; s < USED; ++s) {
          frag_t of[X::PLANES], b[4];
          X::pack(P + s * X::TILES, of);
#pragma unroll
          for (int t = 0; t < 4; ++t) b[t] = X::across(bt, LDB, s, 16 * t, lane);
#pragma unroll
          for (int p = 0; p < X::PLANES; ++p)
#pragma unroll
            for (int t = 0; t < 4; ++t) o[t] = M::mma(b[t], of[p], o[t]);
        }
      };
      if (__builtin_amdgcn_readfirstlane(special)) {       // a row of b holds an infinity or NaN, whose product with 0 is not 0: rows one at a time, each to those from itself on
#pragma unroll 1
        for (int j = 0; j < CHUNK; ++j) {
          float p = 0.f;
#pragma unroll
          for (int s = 0; s < STEPS; ++s) {
            T e[W];
            __builtin_memcpy(e, &x[s], sizeof(e));
#pragma unroll
            for (int i = 0; i < W; ++i) p += Store<T>::load1(e + i) * Store<T>::load1(at + j * LDA + s * M::KSTEP + l4 * W + i);
          }
          p += __shfl_xor(p, 16);
          p += __shfl_xor(p, 32);
          p *= pair_power[CHUNK - 1 - row + j];
#pragma unroll
          for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[t][e] += j <= row ? p * Store<T>::load1(bt + j * LDB + 16 * t + 4 * l4 + e) : 0.f;
        }
      } else if (tile == 0) mix(std::integral_constant<int, 1>());
      else if (tile == 1) mix(std::integral_constant<int, 2>());
      else if (tile == 2) mix(std::integral_constant<int, 3>());
      else mix(std::integral_constant<int, 4>());
      if (r0 + CHUNK < place.rows) request_x(r0 + CHUNK);
      const int c = v0 + 4 * l4;
      if constexpr (VEC) {
        Rows<float, true> to;                              // (offsets in bytes; nothing is written where there is no result)
        to.over(job.out, out_at + r0 * out_step, out_step, out_size);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const unsigned off = row < n && c + 16 * t < V ? to.top + (unsigned)row * to.step + (unsigned)((16 * t + c) * out_size) : NOWHERE;
          if (out_size == 2) __builtin_amdgcn_raw_buffer_store_b64(u32x2_t{f32x2_to_bf16x2(o[t][0], o[t][1]), f32x2_to_bf16x2(o[t][2], o[t][3])}, to.res, off, 0, 0);
          else wide_store(to.res, __builtin_bit_cast(uint4, o[t]), off);
        }
      } else if (job.out && row < n) {
        const long at_row = out_at + (r0 + row) * out_step + c;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (c + 16 * t + e < V) {
              if (out_size == 2) Store<bf16_t>::store1((bf16_t*)job.out + at_row + 16 * t + e, o[t][e]);
              else ((float*)job.out)[at_row + 16 * t + e] = o[t][e];
            }
      }
    }
  }

  float* to = nullptr;
  long rk = job.at_k, rv = job.at_v;
  if (SUM) {
    to = job.pieces + ((size_t)place.piece * g.heads + head) * K * V;
    rk = V; rv = 1;
  } else if (place.segments == 1 && job.state_out && slot >= 0) {
    to = job.state_out + ((size_t)slot * g.heads + head) * K * V;
  }
  if (!to) return;
#pragma unroll
  for (int t = 0; t < DK / 16; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int r = 16 * t + 4 * l4 + e;
      if (r < K && col < V) to[r * rk + col * rv] = S[t][e];
    }
}

// TWO: jobs whose keys are much narrower than the launch's widest (the gradients' walks swap keys and values) walk in tiles of `narrower` columns (777 fp32 rows of 40 x 72: 25 us,
// 29.5 in one width). A kernel of its own: the registers of a walk of 128 columns do not hold both (2 spilled, 3 % of it).
// Two workgroups a compute unit leave 256 registers a lane, which hold every aligned bf16 walk of one width up to 128 columns but not all others (spilled: fp32 of 96 columns 9 at most on whole pieces
// and 40 to 47 on rows that lie anywhere, the 777 rows among them; bf16 rows that lie anywhere 1 to 13). Of 256 columns fp32 walks spill 12 to 50 of the 512 that one workgroup leaves.
constexpr int narrower(int DK) { return DK <= 64 ? 32 : DK <= 128 ? 64 : DK / 2; }
template <typename T, int DK, int PLANES, bool VEC, bool SUM, bool TWO>
__global__ __launch_bounds__(256, DK <= (sizeof(T) == 2 ? 128 : SUM ? 0 : 96) ? 2 : 1) void walk_kernel(LinearArgs g) {
  if (TWO && g.job[blockIdx.y].K <= narrower(DK)) walk<T, TWO ? narrower(DK) : DK, PLANES, VEC, SUM>(g);
  else walk<T, DK, PLANES, VEC, SUM>(g);
}

// The states before each segment from the segments' own, in place, and the last one: a thread four elements (or one, where a state is no whole number of fours), segments
// in order
template <int E>
__global__ __launch_bounds__(256) void scan_kernel(LinearArgs g, int blocks) {
  typedef float vec_t __attribute__((ext_vector_type(E)));
  const LinearJob job = g.job[blockIdx.y];
  const int K = job.K, V = job.V, pair = blockIdx.x / blocks, n = pair / g.heads, head = pair % g.heads;
  int start, length, first;
  if (g.starts) {
    start = clamp_row(g.starts[n], g.rows);
    length = max(0, clamp_row(g.starts[n + 1], g.rows) - start);
    first = g.by_rows ? 2 * start / g.segment : start / g.segment + n;
  } else {
    length = g.rows / g.sequences;
    first = n * max(1, (length + g.segment - 1) / g.segment);
  }
  const int count = (length + g.segment - 1) / g.segment;
  const int i = ((blockIdx.x - pair * blocks) * 256 + threadIdx.x) * E;
  if (count < 2 || i >= K * V) return;                     // (the walk of a single segment has done all of it)
  const float lam = g.log_decay[head];
  int slot = g.slots ? g.slots[n] : n;
  if ((unsigned)slot >= (unsigned)g.pool) slot = -1;
  size_t at[E];
#pragma unroll
  for (int j = 0; j < E; ++j) {
    const int r = (i + j) / V, c = i + j - r * V;
    at[j] = slot >= 0 ? ((size_t)slot * g.heads + head) * K * V + r * job.at_k + c * job.at_v : 0;
  }
  vec_t s;
#pragma unroll
  for (int j = 0; j < E; ++j) s[j] = job.state_in && slot >= 0 ? job.state_in[at[j]] : 0.f;
  const float keep = expf((float)g.segment * lam), keep_last = expf((float)(length - (count - 1) * g.segment) * lam);
  float* p = job.pieces + ((size_t)first * g.heads + head) * K * V + i;
  const size_t step = (size_t)g.heads * K * V;
  constexpr int AHEAD = 8;
  for (int k0 = 0; k0 < count; k0 += AHEAD) {
    vec_t own[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) own[k] = *reinterpret_cast<const vec_t*>(p + (size_t)min(k0 + k, count - 1) * step);
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      if (k0 + k >= count) break;
      *reinterpret_cast<vec_t*>(p + (size_t)(k0 + k) * step) = s;
      s = (k0 + k + 1 == count ? keep_last : keep) * s + own[k];
    }
  }
  if (!job.state_out || slot < 0) return;
#pragma unroll
  for (int j = 0; j < E; ++j) job.state_out[at[j]] = s[j];
}

// Sums over the heads that share keys and values: a workgroup a row, of the keys' gradients or of the values'
template <typename T> __global__ __launch_bounds__(256) void share_kernel(LinearShareArgs a) {
  const LinearShareArgs::One one = a.of[blockIdx.y];
  const int r = blockIdx.x;
  if (a.starts && (r < a.starts[0] || r >= a.starts[a.sequences])) return;
  const float* p = one.in + (size_t)r * a.groups * a.share * one.cols;
  for (int i = threadIdx.x; i < a.groups * one.cols; i += 256) {
    const int h = i / one.cols, c = i - h * one.cols;
    float t = 0.f;
    for (int k = 0; k < a.share; ++k) t += p[(size_t)(h * a.share + k) * one.cols + c];
    Store<T>::store1((T*)one.out + (size_t)r * one.ld + i, t);
  }
}

// ---- one row of every sequence -------------------------------------------------------------------

// S <- g S + k v^T, o = scale S^T q. A workgroup a sequence and head: COLS threads for four columns of S each, 256 / COLS rows at a time; all of a thread's rows are requested before the
// first one is needed. Bound by memory: S is read and written once (128 requests, 16 heads of 128: 46.5 us, 5.8 TB/s; 61.6 with stores through the caches).
template <typename T, int COLS, int ROWS, bool VEC>
__global__ __launch_bounds__(256) void step_kernel(LinearStepArgs a) {
  constexpr int PAR = 256 / COLS;
  __shared__ float q[LINEAR_DIM_MAX], k[LINEAR_DIM_MAX];
  __shared__ float4 red[PAR][COLS];
  const int n = blockIdx.x / a.heads, head = blockIdx.x - n * a.heads, K = a.K, V = a.V, tid = threadIdx.x;
  const int c = tid % COLS * 4, p = tid / COLS;
  int slot = a.slots ? a.slots[n] : n;
  if ((unsigned)slot >= (unsigned)a.pool) slot = -1;
  const size_t at = slot >= 0 ? ((size_t)slot * a.heads + head) * K * V : 0;
  const float* in = a.state_in && slot >= 0 ? a.state_in + at : nullptr;
  float* out = a.state_out && slot >= 0 ? a.state_out + at : nullptr;
  auto load = [&](int r) __attribute__((always_inline)) {
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (in && r < K) {
      const float* f = in + (size_t)r * V + c;
      if (VEC) { if (c < V) s = *reinterpret_cast<const float4*>(f); }
      else {
        if (c < V) s.x = f[0];
        if (c + 1 < V) s.y = f[1];
        if (c + 2 < V) s.z = f[2];
        if (c + 3 < V) s.w = f[3];
      }
    }
    return s;
  };
  float4 S[ROWS];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) S[i] = load(p + i * PAR);
  for (int i = tid; i < K; i += 256) {
    q[i] = Store<T>::load1((const T*)a.q + (size_t)n * a.ld_q + (size_t)head * K + i);
    k[i] = Store<T>::load1((const T*)a.k + (size_t)n * a.ld_k + (size_t)(head / a.share) * K + i);
  }
  float v[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = c + j < V ? Store<T>::load1((const T*)a.v + (size_t)n * a.ld_v + (size_t)(head / a.share) * V + c + j) : 0.f;
  const float keep = expf(a.log_decay[head]);
  __syncthreads();
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int r0 = 0; r0 < K; r0 += ROWS * PAR) {
    if (r0) {
#pragma unroll
      for (int i = 0; i < ROWS; ++i) S[i] = load(r0 + p + i * PAR);
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      const int r = r0 + p + i * PAR;
      if (r >= K) continue;
      const float kr = k[r], qr = q[r];
      float4 s = S[i];
      s.x = keep * s.x + kr * v[0]; s.y = keep * s.y + kr * v[1]; s.z = keep * s.z + kr * v[2]; s.w = keep * s.w + kr * v[3];
      o.x += qr * s.x; o.y += qr * s.y; o.z += qr * s.z; o.w += qr * s.w;
      if (out) {
        float* f = out + (size_t)r * V + c;
        if (VEC) { if (c < V) put16(reinterpret_cast<float4*>(f), s, a.past); }
        else {
          if (c < V) f[0] = s.x;
          if (c + 1 < V) f[1] = s.y;
          if (c + 2 < V) f[2] = s.z;
          if (c + 3 < V) f[3] = s.w;
        }
      }
    }
  }
  red[p][tid % COLS] = o;
  __syncthreads();
  for (int i = tid; i < V; i += 256) {
    float t = 0.f;
#pragma unroll
    for (int j = 0; j < PAR; ++j) t += reinterpret_cast<const float*>(&red[j][0])[i];
    Store<T>::store1((T*)a.o + (size_t)n * a.ld_o + (size_t)head * V + i, a.scale * t);
  }
}

template <typename T, int DK, int PLANES, bool VEC, bool SUM, bool TWO> hipError_t walk_run(const LinearArgs& g, int jobs, hipStream_t s) {
  constexpr int LDA = DK + Mix<T>::PAD, LDB = SLICE + Mix<T>::PAD;
  constexpr size_t lds = (size_t)(CHUNK * LDA + CHUNK * LDB + (SUM ? 0 : Mix<T>::PLANES * SLICE * DK)) * sizeof(T);
  static const hipError_t allowed = hipFuncSetAttribute((const void*)walk_kernel<T, DK, PLANES, VEC, SUM, TWO>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (allowed != hipSuccess) return allowed;
  int slices = 0;
  for (int j = 0; j < jobs; ++j) slices = g.job[j].slices > slices ? g.job[j].slices : slices;
  DDG_LAUNCH((walk_kernel<T, DK, PLANES, VEC, SUM, TWO>), dim3((unsigned)(g.segments * g.heads * slices + 7) / 8 * 8, jobs), dim3(256), lds, s, g);
  return hipGetLastError();
}
template <typename T, int DK, int PLANES, bool VEC, bool SUM> hipError_t walk_widths(const LinearArgs& g, int jobs, hipStream_t s) {
  bool two = false;
  for (int j = 0; j < jobs; ++j) two |= g.job[j].K <= narrower(DK);
  if constexpr (DK > 32) if (two) return walk_run<T, DK, PLANES, VEC, SUM, true>(g, jobs, s);
  return walk_run<T, DK, PLANES, VEC, SUM, false>(g, jobs, s);
}
template <typename T, int DK, bool VEC, bool SUM> hipError_t walk_planes(const LinearArgs& g, int jobs, hipStream_t s) {
  if constexpr (sizeof(T) == 4) {
    return walk_widths<T, DK, 1, VEC, SUM>(g, jobs, s);
  } else {
    bool kept = false;
    for (int j = 0; j < jobs; ++j) kept |= g.job[j].state_out != nullptr;
    return kept ? walk_widths<T, DK, 3, VEC, SUM>(g, jobs, s) : walk_widths<T, DK, 2, VEC, SUM>(g, jobs, s);
  }
}
template <typename T, bool VEC, bool SUM> hipError_t walk_any(const LinearArgs& g, int jobs, hipStream_t s) {
  int most = 0;
  for (int j = 0; j < jobs; ++j) most = g.job[j].K > most ? g.job[j].K : most;
  if (most <= 32) return walk_planes<T, 32, VEC, SUM>(g, jobs, s);
  if (most <= 64) return walk_planes<T, 64, VEC, SUM>(g, jobs, s);
  if (most <= 96) return walk_planes<T, 96, VEC, SUM>(g, jobs, s);
  if (most <= 128) return walk_planes<T, 128, VEC, SUM>(g, jobs, s);
  if (most <= 192) return walk_planes<T, 192, VEC, SUM>(g, jobs, s);
  return walk_planes<T, 256, VEC, SUM>(g, jobs, s);
}
// Pieces of 16 bytes, and a chunk of rows inside the 31 bits of an offset
bool whole(const void* p, long ld, int dim, size_t size) {
  return (uintptr_t)p % 16 == 0 && (size_t)ld * size % 16 == 0 && (size_t)dim * size % 16 == 0 && (size_t)ld * size < (1u << 31) / CHUNK;
}
template <typename T> hipError_t walk_typed(const LinearArgs& g, int jobs, hipStream_t s) {
  bool vec = true;
  for (int i = 0; i < jobs; ++i) {
    const LinearJob& j = g.job[i];
    vec &= whole(j.x, j.ld_x, j.K, sizeof(T)) && whole(j.a, j.ld_a, j.K, sizeof(T)) && whole(j.b, j.ld_b, j.V, sizeof(T)) &&
           whole(j.out, j.ld_out, j.V, j.out_f32 ? 4 : sizeof(T));
  }
  if (g.split) {
    hipError_t e = vec ? walk_any<T, true, true>(g, jobs, s) : walk_any<T, false, true>(g, jobs, s);
    if (e != hipSuccess) return e;
    int most = 0;
    bool fours = true;
    for (int i = 0; i < jobs; ++i) {
      const int cells = g.job[i].K * g.job[i].V;
      most = cells > most ? cells : most;
      fours &= cells % 4 == 0;
    }
    const int each = fours ? 1024 : 256, blocks = (most + each - 1) / each;
    if (fours) DDG_LAUNCH(scan_kernel<4>, dim3(blocks * g.sequences * g.heads, jobs), dim3(256), 0, s, g, blocks);
    else DDG_LAUNCH(scan_kernel<1>, dim3(blocks * g.sequences * g.heads, jobs), dim3(256), 0, s, g, blocks);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return vec ? walk_any<T, true, false>(g, jobs, s) : walk_any<T, false, false>(g, jobs, s);
}

template <typename T, int COLS, int ROWS> hipError_t step_run(const LinearStepArgs& a, bool vec, hipStream_t s) {
  if (vec) DDG_LAUNCH((step_kernel<T, COLS, ROWS, true>), dim3(a.rows * a.heads), dim3(256), 0, s, a);
  else DDG_LAUNCH((step_kernel<T, COLS, ROWS, false>), dim3(a.rows * a.heads), dim3(256), 0, s, a);
  return hipGetLastError();
}
template <typename T> hipError_t step_typed(const LinearStepArgs& given, hipStream_t s) {
  LinearStepArgs a = given;
  a.past = a.state_out && (size_t)a.rows * a.heads * a.K * a.V * 4 > CACHED;
  const bool vec = a.V % 4 == 0 && (uintptr_t)a.state_in % 16 == 0 && (uintptr_t)a.state_out % 16 == 0;
  if (a.V <= 64) return step_run<T, 16, 8>(a, vec, s);
  if (a.V <= 128) return step_run<T, 32, 16>(a, vec, s);
  return step_run<T, 64, 16>(a, vec, s);
}

}  // namespace

// Two workgroups a compute unit are resident: fewer walks than that are cut, for as many (a prompt of 16384 rows, 16 heads of 128, bf16: 134 us in segments of 1024 rows, 145 of 512, 170
// of 2048). A segment costs three passes over a state, so the shortest is three chunks (3010 ragged rows of 12 heads, 64 x 128: 32 us, 36 with two chunks, 41 with one; 70 uncut), of fp32,
// whose chunks take longer, one (777 ragged rows, gradients: 42 us, 58 with two, 90 uncut). Nobody knows how long the longest of ragged sequences is: 2048 rows are the most.
int linear_segment(int rows, int sequences, int walks, bool ragged, int dtype) {
  const int length = ragged ? rows : rows / sequences, average = rows / sequences, least = dtype == BF16 ? 3 * CHUNK : CHUNK;
  const long have = (long)sequences * walks, most = have < 512 ? (512 + have - 1) / have : 1;     // segments of a sequence of average length
  int segment = ((int)((average + most - 1) / most) + CHUNK - 1) / CHUNK * CHUNK;
  segment = segment < least ? least : segment;
  if (ragged && segment > 2048) segment = 2048;
  return length <= segment || (!ragged && most == 1) ? 0 : segment;
}

hipError_t linear_launch(const LinearArgs& a, int jobs, hipStream_t s) { return a.dtype == BF16 ? walk_typed<bf16_t>(a, jobs, s) : walk_typed<float>(a, jobs, s); }

hipError_t linear_step_launch(const LinearStepArgs& a, hipStream_t s) { return a.dtype == BF16 ? step_typed<bf16_t>(a, s) : step_typed<float>(a, s); }

hipError_t linear_share_launch(const LinearShareArgs& a, int count, hipStream_t s) {
  if (a.dtype == BF16) DDG_LAUNCH(share_kernel<bf16_t>, dim3(a.rows, count), dim3(256), 0, s, a);
  else DDG_LAUNCH(share_kernel<float>, dim3(a.rows, count), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace ddg
