// Softmax cross entropy over a vocabulary without its logits. With hidden states h [T][D], vocabulary rows w [V][D] and z = h w^T,
//   l_i = log sum_j exp z_ij - z_i,t_i,   f = sum_i a_i l_i,   P_ij = a_i (exp(z_ij - lse_i) - [j = t_i]),   dh = P w,   dw = P^T h.
// Three matrix products of one kernel (product_body), a panel of tokens at a time:
//   1. z^T = w h^T, a tile of the vocabulary by tokens. A logit lives in a register only: the tile leaves the maximum m and sum of exp(z - m)
//      of each token over the columns of a wave, and, for gradients, exp(z - m) itself in the operands' type. Vocabulary along the tile's rows, because a lane of
//      the matrix instructions holds 16 rows of one column: a token's maximum and sum are its own arithmetic but for one exchange.
//   2. dh^T = w^T P^T    3. dw^T = h^T P
// and between 1 and 2 a pass that joins a token's maxima and sums and turns exp(z - m) into P in place (two roundings in bf16; the target's p - 1 is formed
// in 32 bits and rounded once, and the factor that all tokens share is applied to the sums in 32 bits). What is kept of the T x V values is a panel's, in the
// operands' type, of bounded size: 6 T V D flops in all, where recomputing the logits of a piece for its gradients would take 8. Tokens without a target are left
// out: the others are gathered first, which costs a copy of h and saves their whole share of the products.
// bf16, 8192 tokens of width 4096 over 131072 entries, 5 % of them without a target: 20.7 to 21.9 ms by the card, 1150 to 1210 TFLOP/s of the others (product 1 1140, 2 1380,
// 3 1220, the pass between 5 TB/s); the library's plain product of 8192^3 reaches 1413. The matrix pipes are busy 85 % of product 2's cycles and the clock has fallen from 2.4 to 1.6 GHz: power bounds it.
// Few tokens are bound by memory: 64 over 65536 entries of width 2048 move 805 MB in 172 us, 4.7 TB/s (w read twice, dw written).
#include "ddg_device.h"
#include "ddg_token.h"

#include <type_traits>

namespace ddg {
namespace {

typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// ---- the product ---------------------------------------------------------------------------------

// out[n][m] = sum_k A(m, k) B(n, k). An operand whose rows run along k (KC) is [rows][k], one whose rows run along the tile is [k][rows].
struct ProductArgs {
  const void* A; const void* B;
  long lda, ldb;
  long plane_a, plane_b;     // SPLIT: bytes from one of an operand's three planes to the next
  int M, N, K;               // K: 16-byte pieces of a KC operand start below it; the other kind's rows end there
  const int* count;          // tokens left over the panels, or null: `dynamic` says which of N (1) and K (2) they bound
  int first, dynamic;        // first token of the panel
  int tiles_m, tiles_n, splits;
  // epilogue 1: exp(z - m), maxima and sums, the target's logit
  void* e; long lde; float2* stat; int stats; const int* target; float* zt;   // stat: [N][stats], one of each wave's columns
  // and where one tile holds the whole vocabulary, the rest of the way to P, if row_loss is there
  float* row_loss; float* lse; const float* weight; int whole;
  // epilogue 2: out[map[n]][m] = scale * sum + prev
  void* out; long ldo; int out_f32; const float* prev; long ldp; const float* scale; const int* map; size_t split_stride;
  struct Total { const int* target; const float* row_loss; const float* weight; int T; float* loss; } total;   // loss null, or of one more workgroup
  int past;                  // dw, in a launch of its own: results go past the caches
  int vec;                   // rows of `out` are pieces of a store: 16 bytes (OUT), 4 elements (SUM). Otherwise pieces wherever they begin, and the row's end one by one
};

// 16 bytes a lane from memory straight to LDS, at `lds` + 16 * lane; lanes at NOWHERE write zeros. Nothing waits here: the load has no output register,
// and whoever reads that LDS waits for the counter first (step_barrier).
__device__ __forceinline__ void to_lds(u32x4 res, unsigned voff, unsigned lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(voff), "s"(res) : "memory");
}
// All but the last PENDING loads of this wave have arrived and every LDS read has been answered, in all waves
template <int PENDING> __device__ __forceinline__ void step_barrier() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(PENDING) : "memory");
}
// 16 or 8 bytes to memory; past the caches: nothing else is driven out of them for these
template <typename V> __device__ __forceinline__ void put(void* to, V v, bool past) {
  if (past) {
    asm volatile("" ::: "memory");       // (without these the compiler makes one ordinary store of the two)
    __builtin_nontemporal_store(v, reinterpret_cast<V*>(to));
    asm volatile("" ::: "memory");
  } else {
    *reinterpret_cast<V*>(to) = v;
  }
}
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
__device__ __forceinline__ u32x4 resource(const void* p) {
  const uint64_t a = (uint64_t)(uintptr_t)p;
  return u32x4{(unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)a), (unsigned)__builtin_amdgcn_readfirstlane((int)((unsigned)(a >> 32) & 0xffffu)),
               0x80000000u, 0x00027000u};
}

template <typename T> struct Frag;
template <> struct Frag<bf16_t> {
  typedef bf16x8_t t;
  __device__ static __forceinline__ f32x16_t mma(t a, t b, f32x16_t c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Frag<float> {
  typedef f32x4_t t;
  // four instructions of k = 2: instruction j contracts element j of both half-waves
  __device__ static __forceinline__ f32x16_t mma(t a, t b, f32x16_t c) {
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
    return c;
  }
};

// One operand's tile of a step in LDS: R rows of the tile by KB bytes of k, 128 or 64.
//   KC: [R][KB bytes], 16-byte piece c of row r at place c ^ f(r), f = r >> 1 & 7 (KB 64: r >> 2 & 3): any 16 neighbouring rows have a fragment's pieces in
//   different banks (two or four rows to the 256 bytes of all banks).
//   else: [BK][R], whose fragments are read transposed; 64-byte pieces (bf16: 32 columns) of row k at place piece ^ (k & 3), so that the four
//   rows of a transposing read lie in different banks (R = 64: two rows to 256 bytes, place ^ (k >> 1 & 1)); fp32: 128-byte pieces, place ^ (k >> 2 & 1).
template <typename T, int R, int KB, bool KC, int NT> struct Operand {
  static constexpr int SZ = sizeof(T), BK = KB / SZ, BYTES = R * KB, ROW = KB / 16, LOADS = R * ROW / NT, RB = R * SZ, PER = RB / 16;
  static_assert(LOADS >= 1 && R * ROW % NT == 0, "every thread loads");
  unsigned off[LOADS];       // bytes from the step's base
  int kpos[KC ? 1 : LOADS];  // k of the loads (KC: of all)
  const unsigned char* base;
  long advance;

  static __device__ __forceinline__ int place(int r) { return KB == 128 ? r >> 1 & 7 : r >> 2 & 3; }
  static __device__ __forceinline__ int swizzle(int k) {    // in 16-byte pieces
    if (SZ == 4) return ((k >> 2) & 1) << 3;
    return RB >= 256 ? (k & 3) << 2 : ((k >> 1) & 1) << 2;
  }
  // rows [r0, r0 + R) of `rows`, from k0 on
  __device__ __forceinline__ void init(const void* p, long ld, int r0, int rows, int k0, int tid) {
    if (KC) {
      static_assert(!KC || NT / ROW % 16 == 0, "one place for all loads of a thread");
      base = (const unsigned char*)p + ((size_t)r0 * ld + k0) * SZ;
      advance = KB;
#pragma unroll
      for (int j = 0; j < LOADS; ++j) {
        const int r = tid / ROW + j * (NT / ROW), c = (tid % ROW) ^ place(r);
        off[j] = r0 + r < rows ? (unsigned)(r * (unsigned)(ld * SZ) + c * 16) : NOWHERE;
      }
      kpos[0] = ((tid % ROW) ^ place(tid / ROW)) * (16 / SZ);
    } else {
      base = (const unsigned char*)p + ((size_t)k0 * ld + r0) * SZ;
      advance = (long)BK * ld * SZ;
#pragma unroll
      for (int j = 0; j < LOADS; ++j) {
        const int q = tid + j * NT, k = q / PER, c = (q % PER) ^ swizzle(k);
        kpos[j] = k;
        off[j] = r0 + c * (16 / SZ) < rows ? (unsigned)(k * (unsigned)(ld * SZ) + c * 16) : NOWHERE;
      }
    }
  }
  // load j of a step's tile, through its resource; `left`: how much of k there is from the step's start on
  __device__ __forceinline__ void load(const u32x4 res, unsigned lds, int wave, int left, int j) const {
    to_lds(res, kpos[KC ? 0 : j] < left ? off[j] : NOWHERE, (unsigned)__builtin_amdgcn_readfirstlane((int)(lds + (wave * 64 + j * NT) * 16)));
  }
  __device__ __forceinline__ void step() { base += advance; }
};

// Fragment reads of a wave: rows [wbase + 32 i, ..), k = 16 s / SZ * 2 ..
template <typename T, int R, int KB, bool KC, int TILES> struct Reader {
  static constexpr int SZ = sizeof(T), RB = R * SZ;
  typedef Operand<T, R, KB, KC, 64> Op;
  unsigned at[KC ? 1 : TILES], flip;
  __device__ __forceinline__ void init(int wbase, int lane) {
    const int l32 = lane & 31, hi = lane >> 5;
    if (KC) {
      at[0] = (wbase + l32) * KB;
      flip = (hi ^ Op::place(l32)) << 4;
    } else if (SZ == 2) {
      const int i = lane & 15, k = hi * 8 + i / 4;
#pragma unroll
      for (int t = 0; t < TILES; ++t) {
        const int byte = (wbase + t * 32 + ((lane >> 4) & 1) * 16 + (i % 4) * 4) * 2;
        at[t] = k * RB + (byte ^ (Op::swizzle(k) << 4));
      }
    } else {
#pragma unroll
      for (int t = 0; t < TILES; ++t) at[t] = hi * 4 * RB + (((wbase + t * 32 + l32) * 4) ^ (hi << 7));
    }
  }
  __device__ __forceinline__ typename Frag<T>::t get(const unsigned char* tile, int t, int s) const {
    if (KC) return *reinterpret_cast<const typename Frag<T>::t*>(tile + at[0] + t * 32 * KB + (flip ^ (s << 5)));
    if constexpr (SZ == 2) {
      typedef short tr4_t __attribute__((ext_vector_type(4)));
      typedef tr4_t __attribute__((address_space(3))) * lds_ptr_t;
      const unsigned char* p = tile + at[t] + s * 16 * RB;
      const uint2 l = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr_t)(p)));
      const uint2 h = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr_t)(p + 4 * RB)));
      return __builtin_bit_cast(typename Frag<T>::t, make_uint4(l.x, l.y, h.x, h.y));
    } else {
      const unsigned char* p = tile + at[t] + s * 8 * RB;
      return typename Frag<T>::t{*(const float*)p, *(const float*)(p + RB), *(const float*)(p + 2 * RB), *(const float*)(p + 3 * RB)};
    }
  }
};

// The loss: the tokens' losses, weighted, in a fixed order and in 64 bits; by the threads of one workgroup
template <int NT> __device__ __forceinline__ void total_loss(const ProductArgs::Total& a, unsigned char* smem) {
  double* red = reinterpret_cast<double*>(smem);
  int* n_red = reinterpret_cast<int*>(red + NT / 64);
  const int tid = threadIdx.x;
  double t = 0.0;
  int n = 0;
#pragma unroll 4
  for (int i = tid; i < a.T; i += NT) {
    const bool has = a.target[i] >= 0;
    const float l = a.row_loss[i], w = a.weight ? a.weight[i] : 1.f;
    t += has ? (double)l * w : 0.0;
    n += has;
  }
  for (int k = 1; k < 64; k <<= 1) { t += __shfl_xor(t, k); n += __shfl_xor(n, k); }
  if ((tid & 63) == 0) { red[tid >> 6] = t; n_red[tid >> 6] = n; }
  __syncthreads();
  if (tid) return;
  t = 0.0; n = 0;
  for (int i = 0; i < NT / 64; ++i) { t += red[i]; n += n_red[i]; }
  *a.loss = (float)(a.weight ? t : t / (n > 0 ? n : 1));
}
__global__ __launch_bounds__(1024) void vocab_total_kernel(ProductArgs::Total a) {
  __shared__ __align__(8) unsigned char smem[256];
  total_loss<1024>(a, smem);
}

// fp32 operands as three bf16 each, x = x0 + x1 + x2 with 8 bits apiece: the six products of two planes that reach 2^-24 of the whole (the others are
// smaller than the rounding of an fp32 product), the smallest first. Six passes at the bf16 rate are faster than one on the
// fp32 matrix instructions where the sums are long (3000 tokens of width 1000 over 30000 entries: 3.3 ms, 4.46 on the fp32 instructions, the same errors against 64 bits).
__device__ constexpr int PLANES[6][2] = {{2, 0}, {1, 1}, {0, 2}, {1, 0}, {0, 1}, {0, 0}};

// Epilogues: EXP (product 1), OUT (results in the operands' type), SUM (through 32 bits: added to earlier sums, or left in fp32)
enum { EXP = 1, OUT = 2, SUM = 3 };

template <typename T, int BM, int BN, int WM, int WN, int KW, int KB, int STAGES, int EPI, bool SPLIT> struct ProductShape {
  typedef std::conditional_t<EPI == SUM || SPLIT, float, T> Staged;
  static constexpr int NT = WM * WN * KW * 64, STAGE = (BM + BN) * KB;
  // the tile on its way out: 32 rows of each wave column at a time, rows 16 bytes apart in the banks
  static constexpr int PITCH = BM * (int)sizeof(Staged) + 16, LEAVING = WN * 32 * PITCH;
  // and the sums of the waves along k on their way together
  static constexpr int JOIN = KW > 1 ? KW * BM * BN * 4 : 0, MOST = LEAVING > JOIN ? LEAVING : JOIN;
  static constexpr int LDS = STAGES * STAGE > MOST ? STAGES * STAGE : MOST;
};

template <typename T, int BM, int BN, int WM, int WN, int KW, int KB, int STAGES, bool AKC, bool BKC, int EPI, bool SPLIT>
__device__ __forceinline__ void product_body(const ProductArgs& a, unsigned block, unsigned char* smem, bool past) {
  typedef ProductShape<T, BM, BN, WM, WN, KW, KB, STAGES, EPI, SPLIT> Shape;
  constexpr int NT = Shape::NT, MT = BM / WM / 32, NTL = BN / WN / 32, BK = KB / (int)sizeof(T), STEPS = KB / 32, STAGE = Shape::STAGE;
  constexpr bool INTERLEAVED = MT * NTL >= 8;
  typedef Operand<T, BM, KB, AKC, NT> OpA;
  typedef Operand<T, BN, KB, BKC, NT> OpB;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kw = wave / (WM * WN), wm = wave % (WM * WN) % WM, wn = wave % (WM * WN) / WM, l32 = lane & 31, hi = lane >> 5;

  int N = a.N, K = a.K;
  if (a.count) {
    int there = *a.count - a.first;
    there = there < 0 ? 0 : there;
    if (a.dynamic == 1) N = there < N ? there : N;
    else K = there < K ? there : K;
  }
  // Workgroups go to the 8 XCDs round-robin: each XCD gets a run of neighbouring tiles, in bands of 8 along n, which share operands in its L2
  const int tiles = a.tiles_m * a.tiles_n, total = tiles * a.splits, xcd = block & 7, q8 = total >> 3, r8 = total & 7;
  if (EPI != EXP && block == (unsigned)total) {
    total_loss<NT>(a.total, smem);
    return;
  }
  int id = q8 * xcd + (xcd < r8 ? xcd : r8) + (block >> 3);
  const int split = id / tiles;
  id -= split * tiles;
  const int band = id / (8 * a.tiles_m), in_band = id - band * 8 * a.tiles_m, wide = a.tiles_n - band * 8 < 8 ? a.tiles_n - band * 8 : 8;
  const int tm = in_band / wide, tn = band * 8 + in_band % wide, m0 = tm * BM, n0 = tn * BN;
  if (n0 >= N) return;

  const int ksteps = (K + BK - 1) / BK, k_lo = (int)((long)ksteps * split / a.splits), k_hi = (int)((long)ksteps * (split + 1) / a.splits);
  OpA la; OpB lb;
  // Where every workgroup has rows of A of its own, each begins at another k: all of them at the same one would read a column of A at a time, whose pieces
  // lie a row apart, in few of the memory's channels (64 tokens over 65536 entries of width 2048: 86 -> 77 us)
  const int turn = EPI == EXP && MT * NTL < 8 && a.tiles_n <= 2 && k_hi > k_lo ? tm % (k_hi - k_lo) : 0;
  la.init(a.A, a.lda, m0, a.M, (k_lo + turn) * BK, tid);
  lb.init(a.B, a.ldb, n0, N, (k_lo + turn) * BK, tid);
  Reader<T, BM, KB, AKC, MT> ra; Reader<T, BN, KB, BKC, NTL> rb;
  ra.init(wm * (BM / WM), lane);
  rb.init(wn * (BN / WN), lane);
  const unsigned lds = (unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;

  int aim[NTL];              // EXP: the targets of this lane's tokens
  if (EPI == EXP) {
#pragma unroll
    for (int j = 0; j < NTL; ++j) {
      const int n = n0 + wn * (BN / WN) + 32 * j + l32;
      aim[j] = n < N ? a.target[a.first + n] : -1;
    }
  }
  f32x16_t acc[MT][NTL];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NTL; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

  constexpr int PER_STEP = OpA::LOADS + OpB::LOADS, AHEAD = STAGES - 1;
  auto load = [&](int left, unsigned stage) __attribute__((always_inline)) {
    const u32x4 res_a = resource(la.base), res_b = resource(lb.base);
#pragma unroll
    for (int j = 0; j < OpA::LOADS; ++j) la.load(res_a, lds + stage * STAGE, wave, left, j);
#pragma unroll
    for (int j = 0; j < OpB::LOADS; ++j) lb.load(res_b, lds + stage * STAGE + OpA::BYTES, wave, left, j);
  };
  // To the next step that is requested: the first one is `turn`, after the last comes k_lo (SPLIT: of the next pair of planes)
  constexpr int PAIRS = SPLIT ? 6 : 1;
  int at_k = k_lo + turn, pair = 0;
  if (SPLIT) { la.base += PLANES[0][0] * a.plane_a; lb.base += PLANES[0][1] * a.plane_b; }
  auto ahead = [&]() __attribute__((always_inline)) {
    la.step(); lb.step();
    if (++at_k == k_hi) {
      at_k = k_lo;
      la.base -= (k_hi - k_lo) * la.advance; lb.base -= (k_hi - k_lo) * lb.advance;
      if (SPLIT && pair < PAIRS - 1) {
        la.base += (PLANES[pair + 1][0] - PLANES[pair][0]) * a.plane_a;
        lb.base += (PLANES[pair + 1][1] - PLANES[pair][1]) * a.plane_b;
        ++pair;
      }
    }
  };
  auto request = [&](unsigned stage) __attribute__((always_inline)) { load(K - at_k * BK, stage); ahead(); };
  if constexpr (INTERLEAVED) {
    // The matrix instructions of a step in a row, and one LDS read of the next k's fragments or one load between each two: a wave never has a burst of
    // others to issue first (product 2 of 4096 tokens of 131072 entries and width 4096: 3.06 ms, 3.29 with the waves in two groups that take turns at LDS and the matrix
    // pipes, 3.53 with the reads of each k before its instructions). Before a step's last k every wave has read all of its stage; there the next
    // step's loads are waited for. Step t requests step t + AHEAD into the stage of step t - 1. Loads past the end of k are made, and write zeros: the counts are constant.
    static_assert(STAGES >= 3 && PER_STEP % STEPS == 0, "");
#pragma unroll
    for (int t = 0; t < AHEAD; ++t) {
      load(t < (k_hi - k_lo) * PAIRS ? K - at_k * BK : 0, t);
      ahead();
    }
    typename Frag<T>::t fa[2][MT], fb[2][NTL];
    step_barrier<(AHEAD - 1) * PER_STEP>();
#pragma unroll
    for (int i = 0; i < MT; ++i) fa[0][i] = ra.get(smem, i, 0);
#pragma unroll
    for (int j = 0; j < NTL; ++j) fb[0][j] = rb.get(smem + OpA::BYTES, j, 0);
    unsigned stage = 0, before = STAGES - 1;
    const int steps = (k_hi - k_lo) * PAIRS;
    for (int t = 0; t < steps; ++t) {
      const unsigned next = stage == STAGES - 1 ? 0 : stage + 1, fill = lds + before * STAGE;
      const u32x4 res_a = resource(la.base), res_b = resource(lb.base);
      const int left = t + AHEAD < steps ? K - at_k * BK : 0;
#pragma unroll
      for (int s = 0; s < STEPS; ++s) {
        const bool last = s == STEPS - 1;
        if (last) step_barrier<(AHEAD - 2) * PER_STEP + PER_STEP * (STEPS - 1) / STEPS>();
        const unsigned char* at = smem + (last ? next : stage) * STAGE;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int q = 0; q < MT * NTL; ++q) {
          constexpr int EVERY = MT * NTL / (MT + NTL);
          acc[q % MT][q / MT] = Frag<T>::mma(fa[s & 1][q % MT], fb[s & 1][q / MT], acc[q % MT][q / MT]);
          if (q % EVERY == 0 && q / EVERY < MT + NTL) {
            const int f = q / EVERY;
            if (f < MT) fa[(s + 1) & 1][f] = ra.get(at, f, last ? 0 : s + 1);
            else fb[(s + 1) & 1][f - MT] = rb.get(at + OpA::BYTES, f - MT, last ? 0 : s + 1);
          }
#pragma unroll
          for (int d = 0; d < PER_STEP; ++d)
            if (d * MT * NTL * STEPS / PER_STEP == s * MT * NTL + q) {
              if (d < OpA::LOADS) la.load(res_a, fill, wave, left, d);
              else lb.load(res_b, fill + OpA::BYTES, wave, left, d - OpA::LOADS);
            }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      ahead();
      before = stage;
      stage = next;
    }
    step_barrier<0>();
  } else {
    // Few instructions a step: several workgroups of a compute unit fill each other's gaps (dw of 64 tokens over 65536 entries, 268 MB written: 56-58 us with
    // three one-stage workgroups of 128 x 128 on a compute unit, 78 with two of two stages, 75 in the largest tiles). Step t waits for its own loads only, and requests those of step
    // t + AHEAD when every wave is past step t - 1, whose stage they fill.
#pragma unroll
    for (int t = 0; t < AHEAD; ++t) if (k_lo + t < k_hi) request(t);
    unsigned stage = 0, next = AHEAD;
    for (int t = k_lo; t < k_hi; ++t) {
      if (STAGES == 1) {     // the stage is one workgroup's of several: they wait in turn
        if (t > k_lo) lds_barrier();
        request(0);
        step_barrier<0>();
      } else if (t + AHEAD < k_hi) {
        step_barrier<(AHEAD > 0 ? AHEAD - 1 : 0) * PER_STEP>();
        request(next);
      } else {
        step_barrier<0>();
      }
      const unsigned char* at = smem + stage * STAGE;
      stage = stage == STAGES - 1 ? 0 : stage + 1;
      next = next == STAGES - 1 ? 0 : next + 1;
      static_assert(STEPS % KW == 0, "");
#pragma unroll
      for (int s0 = 0; s0 < STEPS / KW; ++s0) {
        const int s = KW == 1 ? s0 : s0 * KW + kw;         // (a wave has its share of the k of each step)
        typename Frag<T>::t fa[MT], fb[NTL];
#pragma unroll
        for (int i = 0; i < MT; ++i) fa[i] = ra.get(at, i, s);
#pragma unroll
        for (int j = 0; j < NTL; ++j) fb[j] = rb.get(at + OpA::BYTES, j, s);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int j = 0; j < NTL; ++j) acc[i][j] = Frag<T>::mma(fa[i], fb[j], acc[i][j]);
      }
    }
  }

  if constexpr (KW > 1) {      // the sums of the waves along k, in their order, in all of them: what follows they all do alike
    static_assert(MT == 1 && NTL == 1, "");
    float4* s_acc = reinterpret_cast<float4*>(smem);
    constexpr int WAVES = WM * WN;
    lds_barrier();
#pragma unroll
    for (int g = 0; g < 4; ++g) s_acc[(wave * 4 + g) * 64 + lane] = make_float4(acc[0][0][4 * g], acc[0][0][4 * g + 1], acc[0][0][4 * g + 2], acc[0][0][4 * g + 3]);
    lds_barrier();
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      float4 t = s_acc[(wave % WAVES * 4 + g) * 64 + lane];
#pragma unroll
      for (int q = 1; q < KW; ++q) {
        const float4 u = s_acc[((q * WAVES + wave % WAVES) * 4 + g) * 64 + lane];
        t.x += u.x; t.y += u.y; t.z += u.z; t.w += u.w;
      }
      acc[0][0][4 * g] = t.x; acc[0][0][4 * g + 1] = t.y; acc[0][0][4 * g + 2] = t.z; acc[0][0][4 * g + 3] = t.w;
    }
  }

  // A lane holds column n = l32 of each 32 x 32 tile, rows 8 g + 4 hi + 0..3. Rows of the result leave through LDS, so that a wave's stores are whole lines.
  const int mw = m0 + wm * (BM / WM) + 4 * hi, nw = n0 + wn * (BN / WN) + l32;
  const float scale = EPI != EXP && a.scale ? *a.scale : 1.f;
#pragma unroll
  for (int j = 0; j < NTL; ++j) {
    if (EPI == EXP) {
      const int n = nw + 32 * j;
      if (m0 + BM > a.M) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) if (mw + 32 * i + 8 * (e / 4) + e % 4 >= a.M) acc[i][j][e] = -__builtin_inff();
      }
      const int t = aim[j] < 0 ? -1 : aim[j] - mw;
      float zt = 0.f;
      if (t >= 0 && t < 32 * MT && (t & 4) == 0 && mw + t < a.M) {   // the target is one of this lane's rows
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) zt = t == 32 * i + 8 * (e / 4) + e % 4 ? acc[i][j][e] : zt;
        if (!a.whole) a.zt[a.first + n] = zt;
      }
      float top = -__builtin_inff();
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, acc[i][j][e]);
      top = fmaxf(top, __shfl_xor(top, 32));
      const float from = top == -__builtin_inff() ? 0.f : top;       // all of them -inf, or past the vocabulary: exp gives 0
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          acc[i][j][e] = __expf(acc[i][j][e] - from);
          sum += acc[i][j][e];
        }
      sum += __shfl_xor(sum, 32);
      if (!a.whole) {
        // (a sum of 0 is of -inf alone: with that as its maximum the factor exp(m - lse) of these entries is 0, whatever the log-sum. A NaN sum keeps a finite one)
        if (hi == 0 && n < N) a.stat[(size_t)n * a.stats + tm * WM + wm] = make_float2(sum == 0.f ? top : from, sum);
      } else {
        // The waves of a token put their maxima and sums together: its log-sum, its loss and its row of P, as vocab_row_kernel has them
        float2* s_stat = reinterpret_cast<float2*>(smem);              // [WM][BN]
        float* s_zt = reinterpret_cast<float*>(s_stat + WM * BN);      // [BN]
        const int col = wn * (BN / WN) + 32 * j + l32;
        lds_barrier();
        if (hi == 0) s_stat[wm * BN + col] = make_float2(top, sum);
        if (t >= 0 && t < 32 * MT && (t & 4) == 0 && mw + t < a.M) s_zt[col] = zt;
        lds_barrier();
        float all = -__builtin_inff();
#pragma unroll
        for (int i = 0; i < WM; ++i) all = fmaxf(all, s_stat[i * BN + col].x);
        const float base = all == -__builtin_inff() ? 0.f : all;
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < WM; ++i) {
          const float2 v = s_stat[i * BN + col];
          if (v.y != 0.f) s += v.y * __expf((v.x == -__builtin_inff() ? 0.f : v.x) - base);
        }
        const float lse = base + logf(s), z = aim[j] >= 0 && aim[j] < a.M ? s_zt[col] : __builtin_nanf("");
        const int token = n < N ? (a.map ? a.map[a.first + n] : a.first + n) : 0;
        if (wm == 0 && hi == 0 && n < N) {
          if (a.row_loss) a.row_loss[token] = aim[j] < 0 ? 0.f : lse - z;
          if (a.lse) a.lse[token] = aim[j] < 0 ? 0.f : lse;
        }
        if (a.e) {
          const float share = aim[j] >= a.M ? __builtin_nanf("") : n < N && a.weight ? a.weight[token] / *a.scale : 1.f;
          const float by = __expf((sum == 0.f ? top : from) - lse) * share;        // (entries that are all -inf: 0, whatever the log-sum)
          const float own = (__expf(z - base) / s - 1.f) * share;
#pragma unroll
          for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const int m = 32 * i + 8 * (e / 4) + e % 4;
              acc[i][j][e] = mw + m < a.M ? (t == m ? own : acc[i][j][e] * by) : 0.f;
            }
        }
      }
      if (!a.e) continue;
    }
    typedef typename Shape::Staged S;
    constexpr int V = 16 / (int)sizeof(S), PIECES = BM / V, ROWS = WN * 32, TURNS = (ROWS * PIECES + NT - 1) / NT;
    float4 prev[EPI == SUM ? TURNS : 1];
    if (EPI == SUM && a.prev) {          // requested before the tile goes through LDS
#pragma unroll
      for (int q = 0; q < TURNS; ++q) {
        const int r = (tid + q * NT) / PIECES, n = n0 + (r / 32) * (BN / WN) + 32 * j + r % 32, m = m0 + (tid + q * NT) % PIECES * V;
        prev[q] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (n >= N || m >= a.M) continue;
        const float* from = a.prev + (size_t)n * a.ldp + m;
        if (a.vec) prev[q] = *reinterpret_cast<const float4*>(from);
        else if (m + 4 <= a.M) __builtin_memcpy(&prev[q], from, 16);
        else prev[q] = make_float4(from[0], m + 1 < a.M ? from[1] : 0.f, m + 2 < a.M ? from[2] : 0.f, m + 3 < a.M ? from[3] : 0.f);
      }
    }
    lds_barrier();
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        Store<S>::store4(reinterpret_cast<S*>(smem + (wn * 32 + l32) * Shape::PITCH) + wm * (BM / WM) + 32 * i + 8 * g + 4 * hi, acc[i][j][4 * g] * scale,
                         acc[i][j][4 * g + 1] * scale, acc[i][j][4 * g + 2] * scale, acc[i][j][4 * g + 3] * scale);
    lds_barrier();
#pragma unroll
    for (int q = 0; q < TURNS; ++q) {
      const int at = tid + q * NT, r = at / PIECES, c = at % PIECES;
      const int n = n0 + (r / 32) * (BN / WN) + 32 * j + r % 32, m = m0 + c * V;
      if (n >= N || (ROWS * PIECES % NT != 0 && at >= ROWS * PIECES)) continue;
      const S* from = reinterpret_cast<const S*>(smem + r * Shape::PITCH) + c * V;
      if (EPI == EXP) {
        if (m < a.lde) *reinterpret_cast<uint4*>((S*)a.e + (size_t)n * a.lde + m) = *reinterpret_cast<const uint4*>(from);
        continue;
      }
      if (m >= a.M) continue;
      const size_t to = a.split_stride * split + (size_t)(a.map ? a.map[a.first + n] : n) * a.ldo + m;
      if (EPI == OUT) {
        if (a.vec) {
          put((T*)a.out + to, *reinterpret_cast<const u32x4*>(from), past);
        } else if (m + V <= a.M) {
          __builtin_memcpy((T*)a.out + to, from, 16);
        } else {
#pragma unroll
          for (int e = 0; e < V; ++e) if (m + e < a.M) ((T*)a.out)[to + e] = reinterpret_cast<const T*>(from)[e];
        }
      } else {
        float v[4];
        Store<float>::load4(reinterpret_cast<const float*>(from), v);
        if (a.prev) { v[0] += prev[q].x; v[1] += prev[q].y; v[2] += prev[q].z; v[3] += prev[q].w; }
        if (a.vec) {
          if (a.out_f32) put((float*)a.out + to, f32x4_t{v[0], v[1], v[2], v[3]}, past);
          else put((T*)a.out + to, u32x2{f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3])}, past);
        } else if (m + 4 <= a.M) {
          if (a.out_f32) {
            __builtin_memcpy((float*)a.out + to, v, 16);
          } else {
            const uint2 b = make_uint2(f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3]));
            __builtin_memcpy((T*)a.out + to, &b, 8);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (m + e < a.M) {
              if (a.out_f32) ((float*)a.out)[to + e] = v[e];
              else Store<T>::store1((T*)a.out + to + e, v[e]);
            }
        }
      }
    }
  }
}

extern __shared__ __align__(1024) unsigned char product_lds[];

template <typename T, int BM, int BN, int WM, int WN, int KW, int KB, int STAGES, bool AKC, bool BKC, int EPI, bool SPLIT>
__global__ __launch_bounds__(WM * WN * KW * 64) __attribute__((amdgpu_waves_per_eu(2))) void product_kernel(ProductArgs a) {
  product_body<T, BM, BN, WM, WN, KW, KB, STAGES, AKC, BKC, EPI, SPLIT>(a, blockIdx.x, product_lds, !AKC && !BKC && a.past);
}
// Products 2 (a) and 3 (b) in one launch, where neither of them fills the chip: the first n workgroups have one of them, the one with the longer sums, the others
// the other. (256 fp32 tokens of width 64 over 100 entries: 24.9 us with a launch for each and for the rows of P, 16.8 with this and the vocabulary in one tile.)
template <typename T, int BM, int BN, int WM, int WN, int KB, int STAGES, bool SPLIT>
__global__ __launch_bounds__(WM * WN * 64) __attribute__((amdgpu_waves_per_eu(2))) void product_pair_kernel(ProductArgs a, ProductArgs b, unsigned n, int b_first) {
  const bool second = blockIdx.x >= n;
  const unsigned block = second ? blockIdx.x - n : blockIdx.x;
  if (second == (b_first != 0)) product_body<T, BM, BN, WM, WN, 1, KB, STAGES, false, true, SUM, SPLIT>(a, block, product_lds, false);
  else product_body<T, BM, BN, WM, WN, 1, KB, STAGES, false, false, SUM, SPLIT>(b, block, product_lds, false);
}

// ---- what lies between the products --------------------------------------------------------------

__device__ __forceinline__ float wave_total(float v) {
  v = row_sum16(v);
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// What the products of P are multiplied by in the end, in 32 bits: 1 / count, or the largest weight (P then holds weights relative to it: equal ones are
// not rounded)
__device__ __forceinline__ float share_of(int count, bool weighted, float top) {
  return !weighted ? 1.f / (float)(count > 0 ? count : 1) : top > 0x1p-100f && top < 0x1p100f ? top : 1.f;
}
// Tokens with a target, in order: idx (their places), their targets, pos (place among them, -1 without one); their count and share. One workgroup.
__global__ __launch_bounds__(1024) void vocab_scan_kernel(const int* target, const float* weight, int T, int* idx, int* kept, int* pos, int* count, float* share) {
  __shared__ int s_wave[16];
  __shared__ float s_top[16];
  float top = 0.f;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int before = 0;
  for (int t0 = 0; t0 < T; t0 += 1024) {
    const int t = t0 + tid, y = t < T ? target[t] : -1;
    const uint64_t mask = __ballot(y >= 0);
    if (lane == 0) s_wave[wave] = __popcll(mask);
    __syncthreads();
    int at = before, all = 0;
    for (int i = 0; i < 16; ++i) { if (i < wave) at += s_wave[i]; all += s_wave[i]; }
    at += __popcll(mask & ((1ull << lane) - 1));
    if (t < T) {
      pos[t] = y >= 0 ? at : -1;
      if (y >= 0) {
        idx[at] = t; kept[at] = y;
        if (weight) top = fmaxf(top, fabsf(weight[t]));
      }
    }
    before += all;
    __syncthreads();
  }
  for (int k = 1; k < 64; k <<= 1) top = fmaxf(top, __shfl_xor(top, k));
  if (lane == 0) s_top[wave] = top;
  __syncthreads();
  if (tid) return;
  for (int i = 1; i < 16; ++i) top = fmaxf(top, s_top[i]);
  *count = before;
  *share = share_of(before, weight != nullptr, top);
}

// The planes of four fp32 values, each the rounding of what the earlier ones left; the first one's stops at the largest bf16, which the lowest and highest fp32 values would
// round past to infinity. (Infinities and NaN leave a rest that is neither 0 nor finite: NaN.)
__device__ __forceinline__ void split4(float4 v, uint2 (&p)[3]) {
  float f[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    constexpr float MOST = 0x1.fep127f;
    const auto whole = [&](float x) { return i == 0 ? __builtin_amdgcn_fmed3f(x, -MOST, MOST) : x; };
    p[i] = make_uint2(f32x2_to_bf16x2(whole(f[0]), whole(f[1])), f32x2_to_bf16x2(whole(f[2]), whole(f[3])));
    f[0] -= __uint_as_float(p[i].x << 16); f[1] -= __uint_as_float(p[i].x & 0xffff0000u);
    f[2] -= __uint_as_float(p[i].y << 16); f[3] -= __uint_as_float(p[i].y & 0xffff0000u);
  }
}

// A workgroup a row: row t of `from` to row pos[t] of `to` (pos null: t), widened to a whole number of 16-byte pieces with zeros. Without a place: the
// token's results, which are zeros. Scan: pos is not there yet; each workgroup counts the targets before its token, and leaves what the scan kernel would.
// SPLIT: to three planes of bf16, `plane` elements apart.
struct Scan { const int* target; const float* weight; int T; int* idx; int* kept; int* count; float* share; };
constexpr int SCAN_IN_GATHER = 2048;     // tokens: a workgroup reads up to 8 KB of targets, less than the 4 us that a launch before it takes
template <typename T, bool SPLIT>
__global__ __launch_bounds__(256) void vocab_gather_kernel(const T* from, long ld, int dim, int dim_p, bool vec, const int* pos, Scan scan, void* to_any,
                                                           size_t plane, T* dh, long ld_dh, float* row_loss, float* lse) {
  constexpr int V = Store<T>::VEC;
  __shared__ int s_n[4];
  __shared__ float s_top[4];
  const int t = blockIdx.x, tid = threadIdx.x;
  int j = t;
  if (scan.target) {
    const int y = scan.target[t];
    const bool end = t == scan.T - 1;
    int n = 0;
    float top = 0.f;
    for (int i = tid; i <= t; i += 256) {
      const bool has = scan.target[i] >= 0;
      n += has && i < t;
      if (end && has && scan.weight) top = fmaxf(top, fabsf(scan.weight[i]));
    }
    for (int k = 1; k < 64; k <<= 1) { n += __shfl_xor(n, k); top = fmaxf(top, __shfl_xor(top, k)); }
    if ((tid & 63) == 0) { s_n[tid >> 6] = n; s_top[tid >> 6] = top; }
    __syncthreads();
    n = s_n[0] + s_n[1] + s_n[2] + s_n[3];
    j = y >= 0 ? n : -1;
    if (tid == 0 && y >= 0) { scan.idx[j] = t; scan.kept[j] = y; }
    if (tid == 0 && end) {
      *scan.count = n + (y >= 0);
      *scan.share = share_of(n + (y >= 0), scan.weight != nullptr, fmaxf(fmaxf(s_top[0], s_top[1]), fmaxf(s_top[2], s_top[3])));
    }
  } else if (pos) {
    j = pos[t];
  }
  if (j < 0) {
    if (tid == 0) { row_loss[t] = 0.f; if (lse) lse[t] = 0.f; }
    if (dh) for (int c = tid; c < dim; c += 256) dh[(size_t)t * ld_dh + c] = T{};
    return;
  }
  const T* in = from + (size_t)t * ld;
  for (int c = tid * V; c < dim_p; c += 256 * V) {
    uint4 q;
    if (vec) {
      q = *reinterpret_cast<const uint4*>(in + c);
    } else if (c + V <= dim) {
      __builtin_memcpy(&q, in + c, 16);
    } else {
      T e[V];
#pragma unroll
      for (int i = 0; i < V; ++i) e[i] = c + i < dim ? in[c + i] : T{};
      __builtin_memcpy(&q, e, 16);
    }
    if constexpr (SPLIT) {
      uint2 planes[3];
      split4(__builtin_bit_cast(float4, q), planes);
#pragma unroll
      for (int i = 0; i < 3; ++i) *reinterpret_cast<uint2*>((bf16_t*)to_any + i * plane + (size_t)j * dim_p + c) = planes[i];
    } else {
      *reinterpret_cast<uint4*>((T*)to_any + (size_t)j * dim_p + c) = q;
    }
  }
}

struct RowArgs {
  const float2* stat; int stats, stat_cols;   // [rows][stats]: maxima and sums of columns
  const float* zt; const int* target; const int* idx; const int* count; const float* weight; const float* share;
  int first, rows, V;
  float* row_loss; float* lse;
  void* p; long ld; int chunk;       // gradients: exp(z - m), turned into P; columns of a workgroup
  bf16_t* planes; size_t plane;      // or P goes here, in three planes
};

// The log-sum of a token from its maxima and sums, its loss, and its row of P: a workgroup takes a chunk of the row (blockIdx.x), each of
// them joins the maxima and sums for itself: no launch of its own for that. Bound by memory: 4096 tokens of 131072 entries, 1.07 GB read and written in place, 412 us,
// 5.2 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void vocab_row_kernel(RowArgs a) {
  constexpr int V = Store<T>::VEC;
  __shared__ float red[2][4];
  const int r = blockIdx.y, tid = threadIdx.x;
  if (a.count && a.first + r >= *a.count) return;
  const float2* st = a.stat + (size_t)r * a.stats;
  float top = -__builtin_inff();
  for (int i = tid; i < a.stats; i += 256) {
    const float2 v = st[i];
    top = fmaxf(top, v.y != 0.f ? v.x : -__builtin_inff());      // (a NaN sum counts)
  }
  top = fmaxf(top, __shfl_xor(top, 1)); top = fmaxf(top, __shfl_xor(top, 2)); top = fmaxf(top, __shfl_xor(top, 4));
  top = fmaxf(top, __shfl_xor(top, 8)); top = fmaxf(top, __shfl_xor(top, 16)); top = fmaxf(top, __shfl_xor(top, 32));
  if ((tid & 63) == 0) red[0][tid >> 6] = top;
  __syncthreads();
  top = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
  const int at = a.first + r, token = a.idx ? a.idx[at] : at, y = a.target[at];
  const bool has = y >= 0 && y < a.V;
  const float zt = has ? a.zt[at] : __builtin_nanf("");             // a target past the vocabulary: its loss and its P are NaN, nothing is read for it
  const float from = top == -__builtin_inff() ? 0.f : top;
  float sum = 0.f;
  for (int i = tid; i < a.stats; i += 256) {
    const float2 v = st[i];
    if (v.y != 0.f) sum += v.y * __expf(v.x - from);
  }
  sum = wave_total(sum);
  if ((tid & 63) == 0) red[1][tid >> 6] = sum;
  __syncthreads();
  sum = red[1][0] + red[1][1] + red[1][2] + red[1][3];
  const float lse = from + logf(sum);
  if (blockIdx.x == 0 && tid == 0) {
    if (a.row_loss) a.row_loss[token] = y < 0 ? 0.f : lse - zt;
    if (a.lse) a.lse[token] = y < 0 ? 0.f : lse;
  }
  if (!a.p) return;
  const float share = !has ? __builtin_nanf("") : a.weight ? a.weight[token] / *a.share : 1.f;
  T* row = (T*)a.p + (size_t)r * a.ld;
  const int lo = blockIdx.x * a.chunk, hi = lo + a.chunk < a.ld ? lo + a.chunk : (int)a.ld;
  for (int c = lo + tid * V; c < hi; c += 256 * V) {
    float v[V];
    Store<T>::load_vec(row + c, v);
    const float scale = c < a.V ? __expf(st[c / a.stat_cols].x - lse) * share : 0.f;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      v[e] = c + e < a.V ? v[e] * scale : 0.f;
      if (c + e == y && has) v[e] = (__expf(zt - from) / sum - 1.f) * share;
    }
    if constexpr (sizeof(T) == 4) {
      if (a.planes) {
        uint2 planes[3];
        split4(make_float4(v[0], v[1], v[2], v[3]), planes);
#pragma unroll
        for (int i = 0; i < 3; ++i) *reinterpret_cast<uint2*>(a.planes + i * a.plane + (size_t)r * a.ld + c) = planes[i];
        continue;
      }
    }
    Store<T>::store_vec(row + c, v);
  }
}

// The same for the loss alone of a few tokens, and the loss, in one workgroup: as many waves a token as there are. (A launch for each of the two takes 4 us; this
// one 5, of 1000 maxima and sums. The product before it reads 65 MB of w in 11.9 us, 5.5 TB/s.)
constexpr int FEW_ROWS = 16;
__global__ __launch_bounds__(1024) void vocab_few_kernel(RowArgs a, int waves, float* loss) {
  __shared__ float s_top[16], s_sum[16], s_loss[FEW_ROWS];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = wave / waves, first = (wave % waves) * 64 + lane, step = waves * 64;
  float top = -__builtin_inff(), sum = 0.f;
  if (r < a.rows) {
    const float2* st = a.stat + (size_t)r * a.stats;
    for (int i0 = first; i0 < a.stats; i0 += 8 * step) {       // 8 of them in flight, joined to what there is
      float2 v[8];
      float above = top;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int i = i0 + k * step;
        v[k] = i < a.stats ? st[i] : make_float2(0.f, 0.f);
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) if (v[k].y != 0.f) above = fmaxf(above, v[k].x);
      if (above == -__builtin_inff()) continue;
      sum *= __expf(top - above);
#pragma unroll
      for (int k = 0; k < 8; ++k) if (v[k].y != 0.f) sum += v[k].y * __expf(v[k].x - above);
      top = above;
    }
    float all = top;
    for (int k = 1; k < 64; k <<= 1) all = fmaxf(all, __shfl_xor(all, k));
    sum = wave_total(top == -__builtin_inff() ? 0.f : sum * __expf(top - all));
    if (lane == 0) { s_top[wave] = all; s_sum[wave] = sum; }
  }
  __syncthreads();
  if (r < a.rows && wave % waves == 0 && lane == 0) {
    for (int i = 0; i < waves; ++i) top = i ? fmaxf(top, s_top[wave + i]) : s_top[wave];
    const float from = top == -__builtin_inff() ? 0.f : top;
    sum = 0.f;
    for (int i = 0; i < waves; ++i) sum += s_sum[wave + i] != 0.f ? s_sum[wave + i] * __expf(s_top[wave + i] - from) : 0.f;
    const int y = a.target[r];
    const float lse = from + logf(sum), l = y < 0 ? 0.f : lse - (y < a.V ? a.zt[r] : __builtin_nanf(""));
    if (a.row_loss) a.row_loss[r] = l;
    if (a.lse) a.lse[r] = y < 0 ? 0.f : lse;
    s_loss[r] = l;
  }
  __syncthreads();
  if (tid || !loss) return;
  double t = 0.0;
  int n = 0;
  for (int i = 0; i < a.rows; ++i) if (a.target[i] >= 0) { t += (double)s_loss[i] * (a.weight ? a.weight[i] : 1.f); ++n; }
  *loss = (float)(a.weight ? t : t / (n > 0 ? n : 1));
}

// dh from the parts of the vocabulary, dw from those of the tokens, in their order: rows of `out`, or of those in `map`
struct Parts { const float* part; int splits; size_t stride; int rows; const int* count; int first; const int* map; void* out; long ld; int f32; };
template <typename T>
__global__ __launch_bounds__(256) void vocab_join_kernel(Parts x, Parts y, int dim, const float* scale) {
  const Parts& a = (int)blockIdx.y < x.rows ? x : y;
  const int r = (int)blockIdx.y < x.rows ? blockIdx.y : blockIdx.y - x.rows, c = (blockIdx.x * 256 + threadIdx.x) * 4;
  if (c >= dim || (a.count && a.first + r >= *a.count)) return;
  const int wide = (dim + 3) & ~3;
  float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int s = 0; s < a.splits; ++s) {
    const float4 q = *reinterpret_cast<const float4*>(a.part + s * a.stride + (size_t)r * wide + c);
    v[0] += q.x; v[1] += q.y; v[2] += q.z; v[3] += q.w;
  }
  const size_t at = (size_t)(a.map ? a.map[a.first + r] : a.first + r) * a.ld + c;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (c + e < dim) {
      if (a.f32) ((float*)a.out)[at + e] = v[e] * *scale;
      else Store<T>::store1((T*)a.out + at + e, v[e] * *scale);
    }
}

// ---- launches ------------------------------------------------------------------------------------

// Tiles of the products: rows along m (vocabulary or width) and n, waves along both and along k, bytes of k in a stage, stages of LDS
enum { LARGE, MEDIUM, SHORT, SMALL, HALF, FEW, DEEP, TILE_KINDS };
struct Tile { int bm, bn, wm, wn, kw, kb, stages; };
constexpr Tile TILES[TILE_KINDS] = {{256, 256, 2, 4, 1, 64, 4}, {128, 128, 2, 2, 1, 128, 2}, {128, 128, 2, 2, 1, 128, 1}, {64, 64, 2, 2, 1, 128, 3},
                                     {128, 64, 4, 1, 1, 128, 3}, {128, 32, 4, 1, 1, 128, 4}, {32, 32, 1, 1, 4, 128, 4}};

template <typename T, int KIND, bool AKC, bool BKC, int EPI, bool SPLIT = false>
hipError_t product_run(ProductArgs a, hipStream_t s) {
  constexpr Tile t = TILES[KIND];
  constexpr int LDS = ProductShape<T, t.bm, t.bn, t.wm, t.wn, t.kw, t.kb, t.stages, EPI, SPLIT>::LDS;
  const auto kernel = &product_kernel<T, t.bm, t.bn, t.wm, t.wn, t.kw, t.kb, t.stages, AKC, BKC, EPI, SPLIT>;
  static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
  if (attr != hipSuccess) return attr;
  a.tiles_m = (a.M + t.bm - 1) / t.bm;
  a.tiles_n = (a.N + t.bn - 1) / t.bn;
  if (a.tiles_n == 0) return hipSuccess;
  DDG_LAUNCH(kernel, dim3(a.tiles_m * a.tiles_n * a.splits + (a.total.loss ? 1 : 0)), dim3(t.wm * t.wn * t.kw * 64), LDS, s, a);
  return hipGetLastError();
}

template <typename T, bool AKC, bool BKC, int EPI>
hipError_t product_any(const ProductArgs& a, int kind, hipStream_t s) {
  if constexpr (sizeof(T) == 4) if (kind == LARGE) return product_run<bf16_t, LARGE, AKC, BKC, EPI, true>(a, s);   // three planes an operand
  if constexpr (sizeof(T) == 2) if (kind == LARGE) return product_run<T, LARGE, AKC, BKC, EPI>(a, s);
  if constexpr (AKC && BKC) if (kind == DEEP) return product_run<T, DEEP, AKC, BKC, EPI>(a, s);
  if constexpr (BKC) {
    if (kind == FEW) return product_run<T, FEW, AKC, BKC, EPI>(a, s);
    if (kind == HALF) return product_run<T, HALF, AKC, BKC, EPI>(a, s);
  }
  if constexpr (!BKC) if (kind == SHORT) return product_run<T, SHORT, AKC, BKC, EPI>(a, s);
  if (kind == SMALL) return product_run<T, SMALL, AKC, BKC, EPI>(a, s);
  return product_run<T, MEDIUM, AKC, BKC, EPI>(a, s);
}
// how an epilogue that goes through 32 bits (SUM), or does not, stores its rows
template <typename T> void set_out(ProductArgs& a, size_t dim, bool sum) {
  const size_t piece = sum ? 4 : 8, bytes = piece * (a.out_f32 || sizeof(T) == 4 ? 4 : 2);
  a.vec = dim % piece == 0 && (uintptr_t)a.out % bytes == 0 && a.ldo % piece == 0 && a.split_stride % piece == 0 &&
          (!a.prev || ((uintptr_t)a.prev % 16 == 0 && a.ldp % 4 == 0));
  a.out_f32 = a.out_f32 || sizeof(T) == 4;
}
// results in the operands' type, or in fp32, or added to earlier ones
template <typename T, bool AKC, bool BKC> hipError_t product_out(ProductArgs a, size_t dim, int kind, hipStream_t s) {
  const bool sum = sizeof(T) == 4 || a.out_f32 || a.prev;
  set_out<T>(a, dim, sum);
  if constexpr (sizeof(T) == 4) return product_any<T, AKC, BKC, SUM>(a, kind, s);
  else return sum ? product_any<T, AKC, BKC, SUM>(a, kind, s) : product_any<T, AKC, BKC, OUT>(a, kind, s);
}

template <typename T, int KIND, bool SPLIT = false> hipError_t product_pair_run(ProductArgs a, ProductArgs b, hipStream_t s) {
  constexpr Tile t = TILES[KIND];
  constexpr int LDS = ProductShape<T, t.bm, t.bn, t.wm, t.wn, t.kw, t.kb, t.stages, SUM, SPLIT>::LDS;
  const auto kernel = &product_pair_kernel<T, t.bm, t.bn, t.wm, t.wn, t.kb, t.stages, SPLIT>;
  static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
  if (attr != hipSuccess) return attr;
  unsigned n[2];
  for (ProductArgs* q : {&a, &b}) {
    q->tiles_m = (q->M + t.bm - 1) / t.bm;
    q->tiles_n = (q->N + t.bn - 1) / t.bn;
    n[q == &b] = q->tiles_m * q->tiles_n * q->splits + (q->total.loss ? 1 : 0);
  }
  const int b_first = (long)b.K * a.splits > (long)a.K * b.splits;
  DDG_LAUNCH(kernel, dim3(n[0] + n[1]), dim3(t.wm * t.wn * 64), LDS, s, a, b, n[b_first], b_first);
  return hipGetLastError();
}
template <typename T> hipError_t product_pair(ProductArgs a, ProductArgs b, size_t dim, int kind, hipStream_t s) {
  set_out<T>(a, dim, true);
  set_out<T>(b, dim, true);
  if constexpr (sizeof(T) == 4) if (kind == LARGE) return product_pair_run<bf16_t, LARGE, true>(a, b, s);
  if constexpr (sizeof(T) == 2) if (kind == LARGE) return product_pair_run<T, LARGE>(a, b, s);
  if (kind == MEDIUM) return product_pair_run<T, MEDIUM>(a, b, s);
  return product_pair_run<T, SMALL>(a, b, s);
}

size_t up(size_t v, size_t to) { return (v + to - 1) / to * to; }
int ceil_div(long a, long b) { return (int)((a + b - 1) / b); }

constexpr size_t PANEL_BYTES = ((size_t)1 << 30) + ((size_t)1 << 24);    // of a panel's P: 4096 tokens of a vocabulary of 131072 in bf16, a quarter of what 8192 logits in fp32 take

// A dw of a quarter of the last cache or more goes past the caches: whoever reads it finds little of it there, and w, which the next call reads, would be read while dw is
// driven out (64 tokens over entries of width 2048, back to back: 65536 of them, 268 MB of dw, 210 us through the caches and 162 past them; 32768 90.8 and 88.5;
// 16384 56.7 and 55.6; 1024 tokens over 65536 the same). Where both gradients share a launch it gains nothing, and the choice between the two costs 1 %.
constexpr size_t PAST_BYTES = (size_t)1 << 26;

}  // namespace

void vocab_plan(VocabPlan* p) {
  const size_t size = dtype_size(p->dtype);
  const int vec = 16 / (int)size;
  const bool b16 = size == 2;
  // The tiles, and for the sums of dh and dw (results of any size, long sums) the parts, that take the least time by what the kinds were measured at: us a
  // step of 128 bytes of k with one workgroup on a compute unit, with as many as fit, how many do, and us for the way in and out. fp32 in the largest tiles
  // is in planes: six steps of bf16, of half as many bytes.
  struct Rate { float alone, full; int fit; float ends; };
  static const Rate rates[2][TILE_KINDS] = {
      {{3.6f, 4.9f, 1, 14.f}, {2.0f, 4.1f, 2, 4.f}, {2.6f, 6.2f, 3, 4.f}, {0.66f, 1.65f, 3, 2.f}, {1.1f, 2.05f, 2, 3.f}, {0.66f, 1.17f, 2, 3.f}, {0.25f, 0.6f, 5, 3.f}},
      {{1.0f, 1.45f, 1, 9.f}, {0.68f, 1.0f, 2, 4.f}, {1.3f, 1.35f, 3, 4.f}, {0.28f, 0.7f, 3, 2.f}, {0.37f, 0.88f, 2, 3.f}, {0.29f, 0.65f, 2, 3.f}, {0.2f, 0.5f, 5, 3.f}}};
  enum Sum { LOGITS, DH, DW };
  auto planes_of_p = [&](int kind) { return !b16 && kind == LARGE && p->grads; };   // P in planes: the pass over the rows writes them, for one tile too
  auto step_time = [](const Rate& r, long groups, int here) {      // of `groups` workgroups, `here` on the fullest compute unit
    const float crowded = r.full * here / r.fit;
    return r.fit == 1 ? r.alone + (r.full - r.alone) * groups / 256 : r.alone > crowded ? r.alone : crowded;
  };
  constexpr float LAUNCH = 4.f;
  auto more = [](int q) { return q < 3 ? q + 1 : q & (q - 1) ? q / 3 * 4 : q / 2 * 3; };     // 1, 2, 3, 4, 6, 8, 12, 16 ...
  auto part_time = [](int q, long m, long n) {       // partial sums, written and read; up to 256 MB of them stay in the last cache
    const float bytes = q * (float)m * n * 8.f;
    return bytes / (bytes < 2.4e8f ? 1e7f : 5e6f);
  };
  auto choose = [&](Sum sum, int tokens, int from, int to, int* kind, int* splits) {
    const long m = sum == LOGITS ? p->vocab : p->dim, n = sum == DW ? p->vocab : tokens, k = sum == LOGITS ? p->dim : sum == DH ? p->vocab : tokens;
    const long steps = ceil_div(k * (long)size, 128);
    float best = -1.f;
    *kind = from; *splits = 1;
    for (int c = from; c < to; ++c) {
      if (sum == DW ? c > SMALL : c == SHORT || (sum == DH && c == DEEP)) continue;
      const Rate r = rates[b16][c];
      const long tiles = (long)ceil_div(m, TILES[c].bm) * ceil_div(n, TILES[c].bn);
      for (int q = 1; q <= (sum == LOGITS ? 1 : 64) && (q == 1 || q * 2 <= steps); q = more(q)) {
        const long groups = tiles * q, a_round = 256 * r.fit, last = groups % a_round;
        auto round = [&](long g) {
          if (g == 0) return 0.f;
          const int here = ceil_div(g, 256);                  // workgroups on the fullest compute unit
          return step_time(r, g, here) * ceil_div(steps, q) + r.ends;
        };
        const float t = (groups / a_round) * round(a_round) + round(last) + (q > 1 ? LAUNCH + part_time(q, m, n) : 0.f) +
                        (sum == LOGITS && (m > TILES[c].bm || planes_of_p(c)) ? LAUNCH : 0.f);      // (the vocabulary in one tile: no pass over the rows)
        if (best < 0.f || t < best) { best = t; *kind = c; *splits = q; }
      }
    }
    return best;
  };
  auto choose_all = [&](int tokens, int from, int to) {
    int one;
    float t = choose(LOGITS, tokens, from, to, &p->cfg_z, &one);
    p->pair = false;
    if (p->grads) {
      const float apart = choose(DH, tokens, from, to, &p->cfg_dh, &p->splits) + choose(DW, tokens, from, to, &p->cfg_dw, &p->splits_dw);
      // Both in one launch, in tiles of one kind: the workgroups of the longer sums begin, the others fill what they leave free (one after the other: 1021 tokens of
      // width 776 over 10007 entries 100 us a call, together 90; 4096 of 1024 over 32768 915 and 875; fp32, 512 of 512 over 8192 136 and 127)
      float least = apart;
      for (int c : {LARGE, MEDIUM, SMALL}) {
        if (c < from || c >= to) continue;
        const Rate r = rates[b16][c];
        const long wide = ceil_div(p->dim, TILES[c].bm), steps_h = ceil_div(p->vocab * (long)size, 128), steps_w = ceil_div(tokens * (long)size, 128);
        const long tiles_h = wide * ceil_div(tokens, TILES[c].bn), tiles_w = wide * ceil_div(p->vocab, TILES[c].bn);
        for (int q = 1; q <= 64 && (q == 1 || (q * 2 <= steps_h && tiles_h * q <= 512 * r.fit)); q = more(q))
          for (int w = 1; w <= 64 && (w == 1 || (w * 2 <= steps_w && tiles_w * w <= 256 * r.fit)); w = more(w)) {
            const long all = tiles_h * q + tiles_w * w;
            const int here = all >= 256 * r.fit ? r.fit : ceil_div(all, 256);
            const float step = step_time(r, all < 256 ? all : 256, here);
            const float th = step * ceil_div(steps_h, q) + r.ends, tw = step * ceil_div(steps_w, w) + r.ends;
            const bool dw_first = tw > th;
            const long slots = 256 * here, n1 = dw_first ? tiles_w * w : tiles_h * q, n2 = all - n1, rest = n1 % slots;
            const float t1 = dw_first ? tw : th, t2 = dw_first ? th : tw;
            const long k = ceil_div(n2, slots - rest);      // rounds of the shorter ones beside the last of the longer ones; where that ends first, in its places too
            float tail = rest && k * t2 < t1 ? t1 : k * t2;
            if (rest && k * t2 > t1) {
              const long behind = (long)(t1 / t2), more_places = n2 - (slots - rest) * behind;
              const float after = t1 + ceil_div(more_places, slots) * t2, in_step = ceil_div(n2 + rest * (behind + 1), slots) * t2;
              tail = after < in_step ? after : in_step;
            }
            float both = (n1 / slots) * t1 + tail - LAUNCH;
            if (q > 1 || w > 1) both += LAUNCH;
            if (q > 1) both += part_time(q, p->dim, tokens);
            if (w > 1) both += part_time(w, p->dim, p->vocab);
            if (both < least) {
              least = both;
              p->pair = true;
              p->cfg_dh = p->cfg_dw = c; p->splits = q; p->splits_dw = w;
            }
          }
      }
      t += least;
    }
    return t;
  };
  p->splits = p->splits_dw = 1;
  p->planes = false;
  if (!b16) {                                        // planes: 10 bytes moved for an element of h and w, 8 for one of P
    const float moved = 10.f * p->dim * ((float)p->vocab + p->tokens) + (p->grads ? 8.f * p->tokens * p->vocab : 0.f);
    const float direct = choose_all(p->tokens, MEDIUM, TILE_KINDS);
    p->planes = choose_all(p->tokens, LARGE, MEDIUM) + moved / 4.5e6f + 5.f < direct;
  }
  p->dim_p = (int)up(p->dim, p->planes ? 8 : vec);
  if (p->planes) p->pack_h = p->pack_w = true;
  p->ld_p = (long)up(p->vocab, 64) + 64;           // (rows an odd number of 128 bytes apart where the vocabulary is a power of two)
  p->pack_h = p->grads || p->pack_h || p->tokens > 64;
  const size_t row = p->grads ? p->ld_p * (p->planes ? 10 : size) : (size_t)p->vocab / 4 + 64;
  long most = (long)(PANEL_BYTES / row / 256 * 256);
  if (most < 256) most = 256;
  p->panels = p->tokens > most ? ceil_div(p->tokens, most) : 1;
  p->panel = p->panels > 1 ? (int)up(ceil_div(p->tokens, p->panels), 256) : p->tokens;
  if (p->panels > 1) p->panels = ceil_div(p->tokens, p->panel);
  choose_all(p->panel, p->planes || b16 ? LARGE : MEDIUM, p->planes ? MEDIUM : TILE_KINDS);
  if (p->panels > 1) { p->splits_dw = 1; p->pair = false; }
  p->whole = p->vocab <= TILES[p->cfg_z].bm && !planes_of_p(p->cfg_z);
  p->stat_cols = TILES[p->cfg_z].bm / TILES[p->cfg_z].wm;
  p->stats = ceil_div(p->vocab, TILES[p->cfg_z].bm) * TILES[p->cfg_z].wm;
  p->acc = p->grads && p->panels > 1 && !p->dw_f32 && b16;
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t o = at; at += up(bytes, 256); return o; };
  const size_t T = p->tokens;
  p->o_scalar = take(256);
  p->o_row = take(T * 16);                          // idx, kept targets, places, losses
  p->o_zt = take(T * 4);
  p->o_stat = take((size_t)p->panel * p->stats * 8);
  p->o_p = p->grads ? take((size_t)p->panel * p->ld_p * size) : 0;
  p->o_planes = p->grads && p->planes ? take((size_t)p->panel * p->ld_p * 6) : 0;
  const size_t operand = p->planes ? 6 : size;
  const size_t part = p->splits > 1 ? (size_t)p->splits * p->panel : 0, part_dw = p->splits_dw > 1 ? (size_t)p->splits_dw * p->vocab : 0;
  p->o_part = p->grads ? take(part * up(p->dim, 4) * 4) : 0;
  p->o_part_dw = p->grads ? take(part_dw * up(p->dim, 4) * 4) : 0;
  p->o_acc = p->acc ? take((size_t)p->vocab * up(p->dim, 4) * 4) : 0;
  p->o_h = p->pack_h ? take(T * p->dim_p * operand) : 0;
  p->o_w = p->pack_w ? take((size_t)p->vocab * p->dim_p * operand) : 0;
  p->bytes = at;
}

namespace {

#define TRY(expr)                       \
  do {                                  \
    const hipError_t e_ = (expr);       \
    if (e_ != hipSuccess) return e_;    \
  } while (0)

template <typename T> hipError_t vocab_run(const VocabPlan& p, const VocabArgs& a, hipStream_t s) {
  const size_t size = sizeof(T);
  int* count = (int*)(a.ws + p.o_scalar);
  float* share = (float*)(a.ws + p.o_scalar) + 1;
  int* idx = (int*)(a.ws + p.o_row), *kept = idx + p.tokens, *pos = kept + p.tokens;
  float* row_loss = a.row_loss ? a.row_loss : (float*)(pos + p.tokens);
  float* zt = (float*)(a.ws + p.o_zt);
  float2* stat = (float2*)(a.ws + p.o_stat);
  const unsigned char* h = (const unsigned char*)a.h;
  const void* w = a.w;
  long ld_h = a.ld_h, ld_w = a.ld_w;
  const size_t operand = p.planes ? 2 : size;                       // bytes of an element of a product's operands
  const size_t plane_h = (size_t)p.tokens * p.dim_p, plane_w = (size_t)p.vocab * p.dim_p, plane_p = (size_t)p.panel * p.ld_p;
  auto gather = [&](const T* from, long ld, int n, bool vec, const Scan& scan, const int* at, void* to, size_t plane, T* dh) {
    if constexpr (sizeof(T) == 4) {
      if (p.planes) {
        DDG_LAUNCH((vocab_gather_kernel<T, true>), dim3(n), dim3(256), 0, s, from, ld, p.dim, p.dim_p, vec, at, scan, to, plane, dh, a.ld_dh, row_loss, a.lse);
        return;
      }
    }
    DDG_LAUNCH((vocab_gather_kernel<T, false>), dim3(n), dim3(256), 0, s, from, ld, p.dim, p.dim_p, vec, at, scan, to, plane, dh, a.ld_dh, row_loss, a.lse);
  };
  if (p.pack_h) {
    const bool alone = p.tokens == 0 || p.tokens > SCAN_IN_GATHER;
    if (alone) {
      DDG_LAUNCH(vocab_scan_kernel, dim3(1), dim3(1024), 0, s, a.target, a.weight, p.tokens, idx, kept, pos, count, share);
      TRY(hipGetLastError());
    }
    if (p.tokens) {
      const bool vec = p.dim == p.dim_p && (uintptr_t)a.h % 16 == 0 && ld_h * size % 16 == 0;
      const Scan scan{alone ? nullptr : a.target, a.weight, p.tokens, idx, kept, count, share};
      gather((const T*)a.h, a.ld_h, p.tokens, vec, scan, (const int*)pos, a.ws + p.o_h, plane_h, (T*)a.dh);
      TRY(hipGetLastError());
    }
    h = a.ws + p.o_h; ld_h = p.dim_p;
  }
  if (p.pack_w) {
    const bool vec = p.dim == p.dim_p && (uintptr_t)a.w % 16 == 0 && ld_w * size % 16 == 0;
    gather((const T*)a.w, a.ld_w, p.vocab, vec, Scan{}, (const int*)nullptr, a.ws + p.o_w, plane_w, (T*)nullptr);
    TRY(hipGetLastError());
    w = a.ws + p.o_w; ld_w = p.dim_p;
  }
  const int* bound = p.pack_h ? count : nullptr;
  ProductArgs::Total total{a.target, row_loss, a.weight, p.tokens, a.loss};   // left to the last panel's product of dh, or dw, if there is one
  for (int panel = 0; panel < p.panels; ++panel) {
    const int first = panel * p.panel, rows = p.tokens - first < p.panel ? p.tokens - first : p.panel;
    ProductArgs z{};
    z.A = w; z.lda = ld_w; z.B = h + (size_t)first * ld_h * operand; z.ldb = ld_h; z.plane_a = plane_w * 2; z.plane_b = plane_h * 2; z.M = p.vocab; z.N = rows; z.K = p.dim_p; z.splits = 1;
    z.count = bound; z.first = first; z.dynamic = 1;
    z.e = p.grads ? a.ws + p.o_p : nullptr; z.lde = p.ld_p; z.stat = stat; z.stats = p.stats; z.target = p.pack_h ? kept : a.target; z.zt = zt;
    if (p.whole) { z.whole = 1; z.row_loss = row_loss; z.lse = a.lse; z.weight = a.weight; z.scale = share; z.map = p.pack_h ? idx : nullptr; }
    TRY((product_any<T, true, true, EXP>(z, p.cfg_z, s)));
    if (rows && !p.whole) {
      RowArgs r{};
      r.stat = stat; r.stats = p.stats; r.stat_cols = p.stat_cols; r.zt = zt; r.target = z.target; r.idx = p.pack_h ? idx : nullptr; r.count = bound;
      r.weight = a.weight; r.share = share; r.first = first; r.rows = rows; r.V = p.vocab; r.row_loss = row_loss; r.lse = a.lse;
      if (!p.pack_h && rows <= FEW_ROWS) {
        DDG_LAUNCH(vocab_few_kernel, dim3(1), dim3(1024), 0, s, r, FEW_ROWS / rows, total.loss);
        return hipGetLastError();
      }
      int chunks = 1;
      if (p.grads) {
        r.p = a.ws + p.o_p; r.ld = p.ld_p;
        if (p.planes) { r.planes = (bf16_t*)(a.ws + p.o_planes); r.plane = plane_p; }
        // enough workgroups to fill the chip, none with less than two trips
        const int unit = 2 * 256 * Store<T>::VEC, most = ceil_div(p.ld_p, unit);
        chunks = ceil_div(2048, rows);
        if (chunks > most) chunks = most;
        r.chunk = (int)up(ceil_div(p.ld_p, chunks), Store<T>::VEC * 256);
        chunks = ceil_div(p.ld_p, r.chunk);
      }
      for (int y = 0; y < rows; y += 65535) {       // (a grid's second dimension)
        RowArgs q = r;
        const int n = rows - y < 65535 ? rows - y : 65535;
        q.first += y; q.stat += (size_t)y * q.stats; q.rows = n;
        if (q.p) q.p = (T*)q.p + (size_t)y * q.ld;
        if (q.planes) q.planes += (size_t)y * q.ld;
        DDG_LAUNCH(vocab_row_kernel<T>, dim3(chunks, n), dim3(256), 0, s, q);
        TRY(hipGetLastError());
      }
    }
    if (!p.grads) continue;
    const bool last = panel + 1 == p.panels;
    const void* probs = a.ws + (p.planes ? p.o_planes : p.o_p);
    ProductArgs dh{}, dw{};
    Parts parts{}, parts_dw{};
    if (a.dh && rows) {
      ProductArgs& g = dh;
      g.A = w; g.lda = ld_w; g.B = probs; g.ldb = p.ld_p; g.plane_a = plane_w * 2; g.plane_b = plane_p * 2; g.M = p.dim; g.N = rows; g.K = p.vocab;
      g.count = bound; g.first = first; g.dynamic = 1; g.splits = p.splits;
      if (last) { g.total = total; total.loss = nullptr; }
      if (p.splits > 1) {
        g.out = a.ws + p.o_part; g.ldo = (long)up(p.dim, 4); g.out_f32 = 1; g.split_stride = (size_t)rows * g.ldo;
        parts = Parts{(const float*)g.out, p.splits, g.split_stride, rows, bound, first, idx, a.dh, a.ld_dh, size == 4};
      } else {
        g.out = a.dh; g.ldo = a.ld_dh; g.map = idx; g.scale = share;
      }
    }
    if (a.dw) {
      ProductArgs& g = dw;
      g.A = h + (size_t)first * ld_h * operand; g.lda = ld_h; g.B = probs; g.ldb = p.ld_p; g.plane_a = plane_h * 2; g.plane_b = plane_p * 2;
      g.M = p.dim; g.N = p.vocab; g.K = rows; g.count = bound; g.first = first; g.dynamic = 2; g.splits = p.splits_dw;
      if (last) { g.total = total; total.loss = nullptr; }
      const bool f32 = size == 4 || p.dw_f32;
      if (p.splits_dw > 1) {
        g.out = a.ws + p.o_part_dw; g.ldo = (long)up(p.dim, 4); g.out_f32 = 1; g.split_stride = (size_t)p.vocab * g.ldo;
        parts_dw = Parts{(const float*)g.out, p.splits_dw, g.split_stride, p.vocab, nullptr, 0, nullptr, a.dw, a.ld_dw, f32};
      } else {
        float* sum = p.acc ? (float*)(a.ws + p.o_acc) : (float*)a.dw;
        const long ld_sum = p.acc ? (long)up(p.dim, 4) : a.ld_dw;
        if (panel) { g.prev = sum; g.ldp = ld_sum; }
        g.scale = share;
        g.out_f32 = f32 || !last;
        g.past = last && (size_t)p.vocab * p.dim * (f32 ? 4 : size) >= PAST_BYTES;
        g.out = !last ? (void*)sum : a.dw; g.ldo = !last ? ld_sum : a.ld_dw;
      }
    }
    if (p.pair && dh.out && dw.out) {
      TRY((product_pair<T>(dh, dw, p.dim, p.cfg_dh, s)));
    } else {
      if (dh.out) TRY((product_out<T, false, true>(dh, p.dim, p.cfg_dh, s)));
      if (dw.out) TRY((product_out<T, false, false>(dw, p.dim, p.cfg_dw, s)));
    }
    for (int y = 0; y < parts.rows + parts_dw.rows; y += 65535) {       // (a grid's second dimension)
      Parts one = parts, two = parts_dw;
      const int skip = y < one.rows ? y : one.rows, skip_dw = y - skip;
      one.part += (size_t)skip * up(p.dim, 4); one.first += skip; one.rows -= skip;
      two.part += (size_t)skip_dw * up(p.dim, 4); two.first += skip_dw; two.rows -= skip_dw;
      const int n = one.rows + two.rows < 65535 ? one.rows + two.rows : 65535;
      DDG_LAUNCH(vocab_join_kernel<T>, dim3(ceil_div(p.dim, 1024), n), dim3(256), 0, s, one, two, p.dim, (const float*)share);
      TRY(hipGetLastError());
    }
  }
  if (total.loss) {
    DDG_LAUNCH(vocab_total_kernel, dim3(1), dim3(1024), 0, s, total);
    TRY(hipGetLastError());
  }
  return hipSuccess;
}

}  // namespace

hipError_t vocab_launch(const VocabPlan& p, const VocabArgs& a, hipStream_t s) {
  return p.dtype == BF16 ? vocab_run<bf16_t>(p, a, s) : vocab_run<float>(p, a, s);
}

}  // namespace ddg
