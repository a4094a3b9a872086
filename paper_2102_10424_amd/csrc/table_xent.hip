// Softmax cross-entropy of rows against a table of class vectors, without the
// logits, and its gradients.
//
//   z_vj = scale <h_v, t_j>,  lse_v = log sum_j e^z_vj,  G_vj = e^(z_vj - lse_v) - [j = y_v],
//   dH = f G T,  dT = f G^T H,  f = grad_scale scale / count.
//
// 16-bit operands: three tiled products on the matrix cores.
//   forward   a tile's logits stay in its accumulators; every wave leaves the
//             maximum and the sum of exponentials over its classes for each of
//             its rows, and a second kernel joins them.
//   gradient, bf16   rows piece by piece (all of them where a piece's room allows):
//             the forward product also leaves E_vj = e^(z_vj - r_v) in bf16, r_v the
//             given class's logit.  bf16 has fp32's range, so an r_v far from the
//             row's largest logit will do, and G_v = e^(r_v - lse_v) E_v needs a factor
//             for the row only: dH takes it with the sums, dT with the rows of H.
//             The given class's entries are left out of E: they are most of a
//             gradient, and p - 1 is small where p is known to bf16 only.  dH adds
//             (p - 1) t_y in fp32 at its end, dT the rows (p - 1) h through the
//             learned rows' sums (embed.hip).  Rows whose largest logit is more than 30 from r_v get
//             their E again, from lse_v.  Three products of n C d, no more than there are.
//   gradient, fp16   (whose range would not do) the table piece by piece: the
//             piece's logits again, as G; then its share of dH and its rows of dT.
// E and G are rounded to the operands' type (relative 2^-9 in bf16, 2^-11 in fp16, where
// G is held times 2^15 so that probabilities down to 2^-29 keep all bits), and so are, in bf16, the
// rows of H times their factors, as matrix instructions want it; everything else is fp32.
//
// In bf16 with gradients 8,192 rows of 2,048 against 131,072 classes take 11.4 to 11.9 ms by the card (1,130
// TFLOP/s over the three products), of 1,024 against 50,001 classes 2.48 to 2.52 ms.  The matrix cores are busy 49 to
// 66% and 43 to 58% of the cycles, waves wait 29 to 39% of theirs: the logits' product ends in
// its exponentials with nothing beside them, and dT's 784 tiles of the smaller one are three
// rounds of the card and 16 more.  One row of 1,024 against 131,072 classes: 58 us, the table's bytes
// at 4.7 TB/s.
//
// All products have the result's rows in the lanes and its columns in the
// accumulator's registers: a row's maximum and sum over the classes are then
// sums over registers, and results leave as 16 bytes a lane.  dH and dT
// contract over the slow index of T and H: those operands lie in LDS as they
// do in memory and are transposed by the LDS reads.
//
// fp32 operands (GIST_DTYPE_F32): rows piece by piece through the library's fp32
// products, with one kernel between them that turns a piece's logits into G.
//
// 8-bit operands: forward only.  They travel as bytes and are widened to bf16, which holds every e4m3
// value, in front of the matrix instruction.

#include <algorithm>

#include "elem.cuh"

#define GIST_LAUNCHED(what)                        \
  do {                                             \
    const gist_status s_ = check_launch(what);     \
    if (s_ != GIST_OK) return s_;                  \
  } while (0)

namespace gist {

namespace {

constexpr int kBlock = 256;
constexpr float kL = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr size_t kPieceBytes = size_t{256} << 20;   // G of one piece, or an fp32 piece's logits
constexpr size_t kExpBytes = size_t{1} << 30;       // E of one piece
constexpr int kNoSlot = INT32_MAX;
constexpr float kFar = 30.f;                        // a row's largest logit from its reference
constexpr size_t kPartBytes = size_t{64} << 20;     // fp32 partial results beyond one

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef int intx4 __attribute__((ext_vector_type(4)));
typedef int intx8 __attribute__((ext_vector_type(8)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef int intx4u __attribute__((ext_vector_type(4), aligned(2)));
typedef int intx4w __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float lg2(float x) { return __builtin_amdgcn_logf(x); }

// ---- products -------------------------------------------------------------------------

enum { kStats = 0, kGrad = 1, kPart = 2, kOut = 3, kExp = 4, kAgain = 5 };

// out[n][m] over m < M, n < N: sum over K of P[m][k] Q[n][k].  An operand is
// either rows with K contiguous (ld: bytes from row to row) or, "transposed", K
// rows with its own index contiguous (ld: bytes from one k to the next).
// RP, RQ: rows of the operand that can be read (transposed: values of its own
// index, a multiple of 8); KP, KQ: values of K that can be, of a transposed one.
// What lies behind them is read as the last again: a step's values of K that only
// one operand has must be zero there.
struct Prod {
  const char* P;
  const char* Q;
  int64_t ldp, ldq;
  int64_t M, N, RP, RQ, KP, KQ;
  int tiles_m, tiles_n, steps, slices, len;   // steps: of 128 bytes of K; len: of one slice
  // kStats, kGrad, kExp, kAgain: classes are m (class0 the first), rows are n
  float scale;
  const float* ps;            // 8-bit scales of P's and Q's rows
  const float* qs;
  const int32_t* labels;
  const int32_t* n_dev;
  int64_t row0, class0;
  floatx2* stats;             // [tiles_m NWM][ldstat]: maximum and sum
  int64_t ldstat;
  float* zy;                  // the given class's logit
  const float* lse;           // kGrad; kExp, kAgain: the rows' references r_v
  const int* far;             // kAgain: by 256 rows, whether one of them is far from its first reference
  void* out;                  // kGrad: G, kExp, kAgain: E (16 bits); kPart: fp32 [slice][N][ldo]; kOut: the gradient
  int64_t ldo;
  int add;                    // kPart: add to what is there
  const float* factor;        // kOut
  const float* row_factor;    // kOut: or NULL; then also pm1 T[ids] is added before the factor
  const float* pm1;
  const int32_t* ids;
  const char* T;
  int64_t ldt;
  int out_store;
  const int32_t* slots;       // kOut: or NULL; rows that have one go to rows[slot] instead, in fp32
  float* rows;
  const float* part;          // kOut: or NULL; added (both: leading dimension ldr)
  int64_t ldr;
};

__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

template <int N>
__device__ __forceinline__ void wait_loads() {
  static_assert(N >= 0 && N < 64, "vmcnt");
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// 16 bytes per lane from memory straight to LDS: base + off (per lane) to dst + 16 lane.
// No vector register is written; the caller waits for vmcnt.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_to_lds(unsigned dst, unsigned off, const char* base) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :
               : "s"(dst), "v"(off), "s"(base)
               : "memory", "m0");
}
#pragma clang diagnostic pop

template <int STORE>
struct Frag {          // 16-bit operands: 8 values of K a lane
  intx4 v;
};
template <>
struct Frag<GIST_STORE_E4M3> {   // 32 values of K a lane
  intx8 v;
};

// Eight of a lane's 8-bit values in bf16, which holds all of them.  8-bit matrix instructions lose what
// lies below some 2^-13 of the largest of a few products, 1.6e-5 of the sums' rms whatever
// their depth, and with it log probabilities of short rows their fifth digit; sums of bf16 products are
// fp32's (4e-8).  The price: 4,093 rows of 1,024 against 50,001 classes 385 us, 8-bit
// instructions 280; one row of 2,048 against 131,072 classes 63 and 62.
__device__ __forceinline__ bf16x8 bf16_of(const Frag<GIST_STORE_E4M3>& f, int s) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  union { bf16x8 v; bf16x2 p[4]; } u;
  u.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f.v[2 * s], 1.f, false);
  u.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f.v[2 * s], 1.f, true);
  u.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f.v[2 * s + 1], 1.f, false);
  u.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f.v[2 * s + 1], 1.f, true);
  return u.v;
}

// 16 x 16 blocks: they take half the passes over the accumulators that 32 x 32 ones do, and
// power is what bounds the products (alone, on random bf16 operands, 2,050 TFLOP/s, 32 x 32
// ones 1,810).
template <int STORE>
__device__ __forceinline__ floatx4 mma(const Frag<STORE>& a, const Frag<STORE>& b, floatx4 c) {
  if constexpr (STORE == GIST_STORE_BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a.v), __builtin_bit_cast(bf16x8, b.v), c, 0, 0, 0);
  else if constexpr (STORE == GIST_STORE_F16)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a.v), __builtin_bit_cast(half8, b.v), c, 0, 0, 0);
  else {
#pragma unroll
    for (int s = 0; s < 4; ++s) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf16_of(a, s), bf16_of(b, s), c, 0, 0, 0);
    return c;
  }
}

// One operand's share of a step in LDS, ROWS of its own index by 128 bytes of K.
//  As rows: 128 bytes a row, its 16-byte piece p at p ^ (row / 2 mod 8), which spreads a
//   fragment read (one piece of 16 rows) over the banks.
//  Transposed: 64 k, 2 ROWS bytes each; 32-byte chunk c (16 of its own index) at c ^ f(k),
//   f(k) = k mod 4 + 4 (k / 8 mod 2): half a wave's transposing read takes k .. k + 3 and
//   k + 8 .. k + 11 of one chunk, which this sends to all 64 banks.
template <int ROWS, bool TR>
struct Tile {
  static constexpr int kPieces = TR ? ROWS / 8 : 8;   // 16-byte pieces of a line's row
  // Where lane's 16 bytes of line L (1 KB of the tile, in LDS order) come from; `left`: rows (or,
  // transposed, values of its own index) that are there.
  __device__ __forceinline__ static unsigned offset(int L, int lane, int64_t ld, int64_t left) {
    if constexpr (!TR) {
      const int row = 8 * L + (lane >> 3);
      const int piece = (lane & 7) ^ (row >> 1 & 7);
      return static_cast<unsigned>(min(static_cast<int64_t>(row), left - 1)) * static_cast<unsigned>(ld) + piece * 16;
    } else {
      const int k = L * (64 / kPieces) + lane / kPieces, s = lane % kPieces;
      const int f = (k & 3) | ((k >> 3 & 1) << 2);
      const int piece = ((s >> 1 ^ f) << 1) | (s & 1);
      const int last = static_cast<int>(min(static_cast<int64_t>(kPieces), left / 8)) - 1;
      return static_cast<unsigned>(k) * static_cast<unsigned>(ld) + min(piece, last) * 16;
    }
  }
  // The same of line L + i where only klim values of K are there: what lies behind them is the last
  // again.  k: of line L.
  __device__ __forceinline__ static unsigned limited(unsigned off, int k, int i, int64_t ld, int klim) {
    return off - static_cast<unsigned>(max(k + i * (64 / kPieces) - (klim - 1), 0)) * static_cast<unsigned>(ld);
  }
  // A lane's part of the address of a wave's first block of 16 rows (blk: a multiple of 4), depth 0.
  __device__ __forceinline__ static int base(int lane, int blk) {
    const int i = lane & 15, g = lane >> 4;
    if constexpr (!TR) {
      return (blk * 16 + i) * 128 + (g ^ (i >> 1)) * 16;
    } else {
      const int k = 8 * g + (i >> 2), f = (i >> 2) | ((g & 1) << 2);
      return k * (2 * ROWS) + ((blk ^ f) << 5) + (i & 3) * 8;
    }
  }
  // Fragment of the wave's block x at depth q (32 values of K; 128 of 8 bits).  `at`: a buffer's base
  // and the lane's; what depends on x and q comes by exclusive or and fixed offsets, so that no
  // address but this one takes a register.
  template <int STORE>
  __device__ __forceinline__ static void read(const char* lds, int at, int q, int x, Frag<STORE>& f) {
    if constexpr (TR) {
      typedef __attribute__((address_space(3))) short4v* Ptr;
      const char* p = lds + (at ^ x << 5) + q * (32 * 2 * ROWS);
      const short4v a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Ptr)(const __attribute__((address_space(3))) char*)p);
      const short4v b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (Ptr)(const __attribute__((address_space(3))) char*)(p + 4 * 2 * ROWS));
      f.v = __builtin_bit_cast(intx4, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    } else if constexpr (STORE == GIST_STORE_E4M3) {
      // any two of a row's eight pieces a lane, the same in both operands: g and g + 4
      const intx4 a = *reinterpret_cast<const intx4*>(lds + at + x * 2048);
      const intx4 b = *reinterpret_cast<const intx4*>(lds + (at ^ 64) + x * 2048);
      f.v = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      f.v = *reinterpret_cast<const intx4*>(lds + (at ^ q * 64) + x * 2048);
    }
  }
};

// Four 16-bit values as fp32.
template <int STORE>
__device__ __forceinline__ void load4_16(const char* base, int64_t e, float (&x)[4]) {
  typedef unsigned short us4 __attribute__((ext_vector_type(4), aligned(2)));
  const us4 t = *reinterpret_cast<const us4*>(reinterpret_cast<const unsigned short*>(base) + e);
#pragma unroll
  for (int q = 0; q < 4; ++q) x[q] = widen<STORE>(t[q]);
}

// Four fp32 values to 16 bits, two to a word.
template <int STORE>
__device__ __forceinline__ void pack4(const float (&v)[4], int (&u)[2]) {
#pragma unroll
  for (int h = 0; h < 2; ++h)
    u[h] = static_cast<int>(static_cast<unsigned>(narrow<STORE>(v[2 * h])) |
                            static_cast<unsigned>(narrow<STORE>(v[2 * h + 1])) << 16);
}

// A 16 x 16 block's registers hold, in lane l, columns 4 (l / 16) + 0..3 of row l mod 16.  Two
// neighbouring blocks, packed (a: columns 0..15, b: 16..31), become eight consecutive columns a
// lane: those from col8(l) on.
__device__ __forceinline__ int col8(int lane) { return ((lane >> 4 & 1) << 4) + ((lane >> 5) << 3); }
__device__ __forceinline__ intx4 join8(const int (&a)[2], const int (&b)[2]) {
  intx4 r;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const auto s = __builtin_amdgcn_permlane16_swap(a[h], b[h], false, false);
    r[h] = s[0];
    r[2 + h] = s[1];
  }
  return r;
}

// Rows of these that a label counts for.
__device__ __forceinline__ int64_t rows_real(const Prod& a) { return a.n_dev ? *a.n_dev - a.row0 : a.N; }

// Tiles of 16 WM NWM columns (M) by 16 WN NWN rows (N); NS buffers in LDS of a step each.
//
// A step's MFMAs go by the wave's WM column blocks, WN at a time; behind each of these the block's
// own fragment is read again, for the next depth, and has the time of all others to
// arrive.  The barrier that frees a buffer stands some blocks into the last depth, when that
// depth's fragments have arrived, so that MFMAs that wait for nothing are on both sides of
// it.  The loads of the step that takes the buffer go out behind it, a few after each
// block: together, eight waves' loads would keep the load path (16 cycles each) for half a step.
template <int STORE, int WM, int WN, int NWM, int NWN, int NS, bool PT, bool QT, int EPI>
__global__ __launch_bounds__(64 * NWM * NWN, NS == 2 ? 2 : 1) void product_kernel(Prod a) {
  constexpr int BM = 16 * WM * NWM, BN = 16 * WN * NWN;
  constexpr int LP = BM / 8, LINES = (BM + BN) / 8, WAVES = NWM * NWN, LOADS = LINES / WAVES;
  static_assert(LINES % WAVES == 0, "a wave's loads");
  static_assert(WM % 4 == 0, "blocks are stored two by two");
  constexpr int BUF = (BM + BN) * 128;
  constexpr bool E8 = STORE == GIST_STORE_E4M3;
  constexpr int QN = E8 ? 1 : 2;      // depths of a step
  constexpr int KSTEP = E8 ? 128 : 64;
  using TP = Tile<BM, PT>;
  using TQ = Tile<BN, QT>;
  __shared__ __attribute__((aligned(1024))) char lds[NS][BUF];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / NWN, wn = wave % NWN;
  const unsigned tiles = static_cast<unsigned>(a.tiles_m) * static_cast<unsigned>(a.tiles_n);   // < 2^31
  const unsigned id = static_cast<unsigned>(xcd_remap(blockIdx.x, gridDim.x));
  const int slice = __builtin_amdgcn_readfirstlane(id / tiles);
  const unsigned t = id - slice * tiles;
  // bands of 8 tile columns: what an XCD works on together shares operands
  const unsigned in_bands = 8u * static_cast<unsigned>(a.tiles_n);
  const int band = static_cast<int>(t / in_bands);
  const int in_band = static_cast<int>(t - band * in_bands);
  const int wide = min(8, a.tiles_m - band * 8);
  const int tm = __builtin_amdgcn_readfirstlane(band * 8 + in_band % wide);
  const int tn = __builtin_amdgcn_readfirstlane(in_band / wide);
  if constexpr (EPI == kAgain) {
    if (a.far[static_cast<int64_t>(tn) * BN >> 8] == 0) return;   // the whole workgroup
  }
  const int64_t m0 = static_cast<int64_t>(tm) * BM, n0 = static_cast<int64_t>(tn) * BN;
  const int k0 = slice * a.len;
  const int steps = min(a.len, a.steps - k0);
  const char* const pb = a.P + (PT ? m0 * 2 : m0 * a.ldp);
  const char* const qb = a.Q + (QT ? n0 * 2 : n0 * a.ldq);
  const unsigned lds0 = static_cast<unsigned>(reinterpret_cast<uintptr_t>(
      (__attribute__((address_space(3))) char*)&lds[0][0]));
  // Every wave loads lines of one operand.
  static_assert(!(PT || QT) || LP % LOADS == 0, "a wave's lines");
  const int L0 = wave * LOADS;
  const bool is_p = L0 < LP;
  unsigned off[LOADS];
#pragma unroll
  for (int i = 0; i < LOADS; ++i)
    off[i] = L0 + i < LP ? TP::offset(L0 + i, lane, a.ldp, a.RP - m0) : TQ::offset(L0 + i - LP, lane, a.ldq, a.RQ - n0);
  // The step whose loads are being issued: where its operands begin, and values of K it has.
  const char* sp = nullptr;
  const char* sq = nullptr;
  int kp = KSTEP, kq = KSTEP;
  auto aim = [&](int j) {
    const int64_t k = k0 + j;
    sp = pb + (PT ? k * KSTEP * a.ldp : k * 128);
    sq = qb + (QT ? k * KSTEP * a.ldq : k * 128);
    if constexpr (PT) kp = static_cast<int>(min(static_cast<int64_t>(KSTEP), a.KP - k * KSTEP));
    if constexpr (QT) kq = static_cast<int>(min(static_cast<int64_t>(KSTEP), a.KQ - k * KSTEP));
  };
  auto load = [&](int buf, int i) {
    unsigned o = off[i];
    if constexpr (PT)
      if (is_p && kp < KSTEP) o = TP::limited(o, L0 * (64 / TP::kPieces) + lane / TP::kPieces, i, a.ldp, kp);
    if constexpr (QT)
      if (!is_p && kq < KSTEP) o = TQ::limited(o, (L0 - LP) * (64 / TQ::kPieces) + lane / TQ::kPieces, i, a.ldq, kq);
    load_to_lds(lds0 + buf * BUF + (L0 + i) * 1024, o, L0 + i < LP ? sp : sq);
  };
  floatx4 acc[WM][WN] = {};
#pragma unroll
  for (int j = 0; j < NS; ++j) {
    aim(min(j, steps - 1));   // always NS: the counts below hold
#pragma unroll
    for (int i = 0; i < LOADS; ++i) load(j, i);
  }
  const int fa = TP::base(lane, wm * WM), fb = BM * 128 + TQ::base(lane, wn * WN);
  Frag<STORE> A[WM], B[2][WN];
  auto read_a = [&](int buf, int q, int x) { TP::template read<STORE>(&lds[0][0], fa + buf * BUF, q, x, A[x]); };
  auto read_b = [&](int to, int buf, int q, int y) {
    TQ::template read<STORE>(&lds[0][0], fb + buf * BUF, q, y, B[to][y]);
  };
  wait_loads<LOADS * (NS - 1)>();
  lds_barrier();
#pragma unroll
  for (int y = 0; y < WN; ++y) read_b(0, 0, 0, y);
#pragma unroll
  for (int x = 0; x < WM; ++x) read_a(0, 0, x);
  constexpr int XB = WM / 4;                        // blocks of the last depth before the barrier
  constexpr int GROUPS = QN * WM;                   // of a step; its loads go out in the first half
  constexpr int PER = (2 * LOADS + GROUPS - 1) / GROUPS;
  int buf = 0, next = 1 % NS, freed = 0;
  for (int j = 0; j < steps; j += 2 / QN) {
    // (B has two sets by depth: with one depth a step, two steps a round)
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      constexpr int kOne = QN == 1;
      const int q = kOne ? 0 : u, f = u;
      if (kOne && u == 1 && j + 1 >= steps) break;
      const bool last = q + 1 == QN;
      const int jj = kOne ? j + u : j;
#pragma unroll
      for (int x = 0; x < WM; ++x) {
        if (last && x == XB) {
          // All fragments of step jj are read by this wave and, behind the barrier, by all, so
          // its buffer takes step jj + NS; step jj + 1 has arrived.
          wait_loads<LOADS * (NS - 2)>();
          lds_barrier();
          freed = buf;
          aim(min(jj + NS, steps - 1));   // past the end: the last step again, never used
        }
        const int pos = last && x >= XB ? x - XB : WM - XB + q * WM + x;   // groups since the barrier
        if (pos < WM - XB || jj > 0) {
#pragma unroll
          for (int i = 0; i < LOADS; ++i)
            if (i / PER == pos) load(freed, i);
        }
#pragma unroll
        for (int y = 0; y < WN; ++y) acc[x][y] = mma<STORE>(A[x], B[f][y], acc[x][y]);
        // the next depth's fragments: this block's, and B's one by one
        if (!last) {
          read_a(buf, q + 1, x);
          if (x < WN) read_b(f ^ 1, buf, q + 1, x);
        } else if (x >= XB) {
          if (x == XB) {
#pragma unroll
            for (int z = 0; z < XB; ++z) read_a(next, 0, z);
#pragma unroll
            for (int y = WM - XB; y < WN; ++y) read_b(f ^ 1, next, 0, y);
          }
          read_a(next, 0, x);
          if (x - XB < WN) read_b(f ^ 1, next, 0, x - XB);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      if (last) {
        buf = next;
        next = next + 1 == NS ? 0 : next + 1;
      }
    }
  }
  wait_loads<0>();   // nothing may still be on its way to LDS when the workgroup ends

  const int li = lane & 15, g4 = 4 * (lane >> 4);
  const int64_t mw = m0 + wm * (WM * 16);   // the wave's first column
  constexpr int OPS = E8 ? static_cast<int>(GIST_STORE_BF16) : STORE;
  if constexpr (EPI == kStats || EPI == kGrad || EPI == kExp || EPI == kAgain) {
    const int64_t real = rows_real(a);
    const bool edge = mw + WM * 16 > a.M;
    if constexpr (E8) {      // the classes' scales
#pragma unroll
      for (int x = 0; x < WM; ++x) {
        const int64_t c = mw + x * 16 + g4;
        float s[4];
        load_some<GIST_STORE_F32, 4>(a.ps, c, a.M - c, 0.f, s);
#pragma unroll
        for (int y = 0; y < WN; ++y)
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[x][y][r] *= s[r];
      }
    }
#pragma unroll
    for (int y = 0; y < WN; ++y) {
      const int64_t row = n0 + (wn * WN + y) * 16 + li;
      const bool there = row < a.N;
      float zs = a.scale;
      if (E8 && there) zs *= a.qs[row];
      const int label = there ? a.labels[row] : -1;
      // the label's place among the wave's classes
      const int64_t mine = label >= 0 ? label - (a.class0 + mw) : -1;
      const bool any_label = __any(mine >= 0 && mine < WM * 16);
#pragma unroll
      for (int x = 0; x < WM; ++x)
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[x][y][r] *= zs;
      if constexpr (EPI == kStats || EPI == kExp) {
        if (edge) {
#pragma unroll
          for (int x = 0; x < WM; ++x)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (mw + x * 16 + g4 + r >= a.M) acc[x][y][r] = -__builtin_inff();
        }
      }
      float sum = 0.f, ref = 0.f;
      if constexpr (EPI != kStats) {
        // E, or G, also of rows and classes that only fill up tiles, and of rows without a label: zeros
        const bool used = there && row < real && label >= 0;
        constexpr bool kG = EPI == kGrad;
        constexpr float kHold = kG && STORE == GIST_STORE_F16 ? 32768.f : 1.f;
        if (used) ref = a.lse[row];
        unsigned short* const g = static_cast<unsigned short*>(a.out) + row * a.ldo + mw + col8(lane);
#pragma unroll
        for (int x = 0; x < WM; x += 2) {
          int w[2][2];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float v[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int c = (x + h) * 16 + g4 + r;
              v[r] = ex2((acc[x + h][y][r] - ref) * kL);
              if (EPI == kExp) sum += v[r];
              if (kG && any_label && mine == c) v[r] -= 1.f;
              v[r] *= kHold;
              if (!used || (edge && mw + c >= a.M)) v[r] = 0.f;
            }
            pack4<OPS>(v, w[h]);
          }
          *reinterpret_cast<intx4*>(g + x * 16) = join8(w[0], w[1]);
        }
      }
      if constexpr (EPI == kStats || EPI == kExp) {
        float m = acc[0][y][0];
#pragma unroll
        for (int x = 0; x < WM; ++x)
#pragma unroll
          for (int r = 0; r < 4; ++r) m = fmaxf(m, acc[x][y][r]);
        m = fmaxf(m, __shfl_xor(m, 16, 64));
        m = fmaxf(m, __shfl_xor(m, 32, 64));
        // The sum by E's exponentials, where these are neither too large nor all too small to be told
        // from zero; else by exponentials of their own.
        if (EPI == kStats || __any(!(fabsf(m - ref) < kFar))) {
          ref = m == -__builtin_inff() ? 0.f : m;
          sum = 0.f;
#pragma unroll
          for (int x = 0; x < WM; ++x) {
            float p[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) p[r] = ex2((acc[x][y][r] - ref) * kL);
            sum += (p[0] + p[1]) + (p[2] + p[3]);
          }
        }
        sum += __shfl_xor(sum, 16, 64);
        sum += __shfl_xor(sum, 32, 64);
        // kept relative to the largest
        if (EPI == kExp) sum *= ex2((ref - (m == -__builtin_inff() ? 0.f : m)) * kL);
        const float s = sum;
        if (there && lane < 16) a.stats[(static_cast<int64_t>(tm) * NWM + wm) * a.ldstat + row] = floatx2{m, s};
        if (any_label) {
#pragma unroll
          for (int x = 0; x < WM; ++x)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (mine == x * 16 + g4 + r) a.zy[row] = acc[x][y][r];
        }
      }
    }
  } else if constexpr (EPI == kPart) {
#pragma unroll
    for (int y = 0; y < WN; ++y) {
      const int64_t row = n0 + (wn * WN + y) * 16 + li;
      if (row >= a.N) continue;
      float* const o = static_cast<float*>(a.out) + (slice * a.N + row) * a.ldo + mw + g4;
#pragma unroll
      for (int x = 0; x < WM; ++x) {
        if (mw + x * 16 + g4 >= a.ldo) continue;    // ldo: a multiple of 4
        floatx4* const p = reinterpret_cast<floatx4*>(o + x * 16);
        floatx4 v = acc[x][y];
        if (a.add) v += *p;
        *p = v;
      }
    }
  } else {
    const float f = *a.factor;
#pragma unroll
    for (int y = 0; y < WN; ++y) {
      const int64_t row = n0 + (wn * WN + y) * 16 + li;
      const bool there = row < a.N;
      if (a.row_factor) {
        // a row that takes no part has factor 0, whatever its sums are; a row without a class in the
        // table (a wrong label) has the other term alone
        const float rf = there ? a.row_factor[row] : 0.f;
        const int id = there ? a.ids[row] : -1;
        const float g = id >= 0 ? a.pm1[row] : 0.f;
#pragma unroll
        for (int x = 0; x < WM; ++x) {
          const int64_t c = mw + x * 16 + g4;
          float t4[4] = {};
          if (id >= 0 && c < a.RP) load4_16<OPS>(a.T + id * a.ldt, c, t4);   // RP: a multiple of 64
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[x][y][r] = rf == 0.f ? 0.f : fmaf(g, t4[r], rf * acc[x][y][r]);
        }
      }
      bool there_out = there;
      if constexpr (QT) {
        const int slot = a.slots && there ? a.slots[row] : kNoSlot;
        if (a.part || slot != kNoSlot) {
          there_out = there && slot == kNoSlot;
#pragma unroll
          for (int x = 0; x < WM; ++x) {
            const int64_t c = mw + x * 16 + g4;
            if (!there || c >= a.ldr) continue;    // ldr: a multiple of 4
            if (a.part) acc[x][y] += *reinterpret_cast<const floatx4*>(a.part + row * a.ldr + c);
            if (slot != kNoSlot) *reinterpret_cast<floatx4*>(a.rows + slot * a.ldr + c) = acc[x][y];
          }
        }
      }
#pragma unroll
      for (int x = 0; x < WM; ++x)
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[x][y][r] *= f;
      if (a.out_store == GIST_STORE_F32) {
#pragma unroll
        for (int x = 0; x < WM; ++x) {
          const int64_t c = mw + x * 16 + g4;
          const float v[4] = {acc[x][y][0], acc[x][y][1], acc[x][y][2], acc[x][y][3]};
          if (there_out && c < a.M) store_some<GIST_STORE_F32, 4>(a.out, row * a.ldo + c, a.M - c, v);
        }
      } else {
#pragma unroll
        for (int x = 0; x < WM; x += 2) {
          int w[2][2];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float v[4] = {acc[x + h][y][0], acc[x + h][y][1], acc[x + h][y][2], acc[x + h][y][3]};
            pack4<OPS>(v, w[h]);
          }
          const intx4 v = join8(w[0], w[1]);
          const int64_t c = mw + x * 16 + col8(lane);
          if (!there_out || c >= a.M) continue;
          unsigned short* const o = static_cast<unsigned short*>(a.out) + row * a.ldo + c;
          if (c + 8 <= a.M) {
            *reinterpret_cast<intx4u*>(o) = v;
          } else {
#pragma unroll
            for (int q = 0; q < 8; ++q)
              if (c + q < a.M) o[q] = static_cast<unsigned short>(static_cast<unsigned>(v[q >> 1]) >> (16 * (q & 1)));
          }
        }
      }
    }
  }
}

// ---- around the products ------------------------------------------------------------------

// Rows of any store as 16-bit rows (or bytes as bytes) of `wide` elements, zeros behind d and behind
// n; with labels, rows that are not labelled are zero.  Eight elements a thread.
template <int SRC, int DST>
__global__ __launch_bounds__(kBlock) void copy_rows_kernel(int64_t n, int64_t n_pad, int d, int wide, const void* __restrict__ x,
                                                           int64_t ldx, void* __restrict__ y,
                                                           const int32_t* __restrict__ labels,
                                                           const int32_t* __restrict__ n_dev) {
  const int per = wide / 8;
  const int64_t count = n_pad * per;
  const int64_t real = n_dev ? max(0, *n_dev) : n;
  for (int64_t e = blockIdx.x * static_cast<int64_t>(kBlock) + threadIdx.x; e < count;
       e += static_cast<int64_t>(gridDim.x) * kBlock) {
    const int64_t row = e / per;
    const int c = static_cast<int>(e - row * per) * 8;
    const bool live = row < n && (!labels || (row < real && labels[row] >= 0));
    if constexpr (DST == GIST_STORE_E4M3) {
      const unsigned char* p = static_cast<const unsigned char*>(x) + row * ldx + c;
      unsigned u[2] = {};
      if (live) {
#pragma unroll
        for (int q = 0; q < 8; ++q)
          if (c + q < d) u[q >> 2] |= static_cast<unsigned>(p[q]) << (8 * (q & 3));
      }
      unsigned* const o = reinterpret_cast<unsigned*>(static_cast<unsigned char*>(y) + row * wide + c);
      o[0] = u[0];
      o[1] = u[1];
    } else {
      float v[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) v[q] = 0.f;
      if (live) {
        if constexpr (SRC == GIST_STORE_F32) {
#pragma unroll
          for (int h = 0; h < 8; h += 4) {
            float t[4];
            load_some<SRC, 4>(x, row * ldx + c + h, d - c - h, 0.f, t);
#pragma unroll
            for (int q = 0; q < 4; ++q) v[h + q] = t[q];
          }
        } else {
          load_some<SRC, 8>(x, row * ldx + c, d - c, 0.f, v);
        }
      }
      store_as<DST, 8>(y, row * wide + c, v);
    }
  }
}

// Joins the maxima and sums of rows row0 ..  (all arrays begin there): ROWS rows a workgroup,
// the others of its threads over the parts.  lse, and the given class's log probability (0
// without one).
template <int ROWS>
__global__ __launch_bounds__(1024) void join_stats_kernel(int64_t row0, int64_t n, int64_t C, int parts, const floatx2* __restrict__ stats,
                                                          int64_t ldstat, const float* __restrict__ zy,
                                                          const int32_t* __restrict__ labels,
                                                          const int32_t* __restrict__ n_dev, float* __restrict__ lse,
                                                          float* __restrict__ lse_out, float* __restrict__ logp,
                                                          float* __restrict__ logp_out, float* __restrict__ ref,
                                                          float* __restrict__ row_factor, int* __restrict__ far) {
  constexpr int G = 1024 / ROWS;
  __shared__ float sm[G][ROWS], ss[G][ROWS];
  const int r = threadIdx.x % ROWS, g = threadIdx.x / ROWS;
  const int64_t row = blockIdx.x * static_cast<int64_t>(ROWS) + r;
  float m = -__builtin_inff(), s = 0.f;
  auto take = [&](float pm, float ps) {
    const float w = fmaxf(m, pm), ref = w == -__builtin_inff() ? 0.f : w;
    s = s * ex2((m - ref) * kL) + ps * ex2((pm - ref) * kL);
    m = w;
  };
  if (row < n) {
    int p = g;
    for (; p + 3 * G < parts; p += 4 * G) {
      floatx2 v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = stats[static_cast<int64_t>(p + i * G) * ldstat + row];
#pragma unroll
      for (int i = 0; i < 4; ++i) take(v[i][0], v[i][1]);
    }
    for (; p < parts; p += G) {
      const floatx2 v = stats[static_cast<int64_t>(p) * ldstat + row];
      take(v[0], v[1]);
    }
  }
  sm[g][r] = m;
  ss[g][r] = s;
  __syncthreads();
  for (int h = G / 2; h > 0; h >>= 1) {
    if (g < h) {
      take(sm[g + h][r], ss[g + h][r]);
      sm[g][r] = m;
      ss[g][r] = s;
    }
    __syncthreads();
  }
  if (g != 0 || row >= n) return;
  const float ls = lg2(s) * kLn2, l = m + ls;
  lse[row] = l;
  if (lse_out) lse_out[row] = l;
  const int y = !n_dev || row0 + row < *n_dev ? labels[row] : -1;
  const float lp = y < 0 ? 0.f : y >= C ? __builtin_nanf("") : zy[row] - m - ls;
  logp[row] = lp;
  if (logp_out) logp_out[row] = lp;
  if (!ref) return;
  // What E needs: the row's factor e^(r - lse) (0: no part in the gradients), and whether its reference was too
  // far off; then E comes again, from lse, and its given class after it.
  float f = 0.f;
  if (y >= 0) {
    if (fabsf(m - ref[row]) > kFar) {
      far[row >> 8] = 1;
      ref[row] = l;
    }
    f = ex2((ref[row] - l) * kL);
  }
  row_factor[row] = f;
}

// The given classes: out of E; p - 1 and the class of every row that takes part (0 and -1 of others).
__global__ __launch_bounds__(kBlock) void given_kernel(int64_t row0, int64_t n, int64_t C, const float* __restrict__ logp,
                                                       const int32_t* __restrict__ labels, const int32_t* __restrict__ n_dev,
                                                       unsigned short* __restrict__ E, int64_t ldE, float* __restrict__ pm1,
                                                       int32_t* __restrict__ ids, int* __restrict__ slots) {
  const int64_t row = blockIdx.x * static_cast<int64_t>(kBlock) + threadIdx.x;
  if (row >= n) return;
  const int y = !n_dev || row0 + row < *n_dev ? labels[row] : -1;
  const bool live = y >= 0 && y < C;
  if (live) E[row * ldE + y] = 0;
  pm1[row] = live ? expm1f(logp[row]) : 0.f;
  ids[row] = live ? y : -1;
  if (slots && live) atomicMin(slots + y, static_cast<int>(row));   // a class's slot: the first of its rows
}

// The rows that have been kept in fp32, by the first of a class's rows: rounded to the gradient's store.
template <int STORE>
__global__ __launch_bounds__(kBlock) void given_out_kernel(int64_t n, int d, const int32_t* __restrict__ ids,
                                                           const int32_t* __restrict__ slot_ids, const float* __restrict__ rows,
                                                           int64_t ldr, const float* __restrict__ factor, void* __restrict__ out,
                                                           int64_t ldo) {
  const int64_t row = blockIdx.x;
  if (slot_ids[row] != row) return;
  const float f = *factor;
  const int64_t o = static_cast<int64_t>(ids[row]) * ldo;
  for (int c = threadIdx.x * 4; c < d; c += kBlock * 4) {
    const floatx4 v = *reinterpret_cast<const floatx4*>(rows + row * ldr + c);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float x[1] = {v[q] * f};
      if (c + q < d) store_as<STORE, 1>(out, o + c + q, x);
    }
  }
}

// Rows of H (bf16, `wide` elements) times their factors, in bf16 with zeros behind the last (and where
// the factor is 0, whatever the row holds): dT's operand.  And times p - 1, in fp32.  With
// slots, also every row's.  Eight elements a thread.
__global__ __launch_bounds__(kBlock) void factored_kernel(int64_t n, int64_t n_pad, int64_t wide, const char* __restrict__ H,
                                                          int64_t ldh, const float* __restrict__ factor, char* __restrict__ F,
                                                          const float* __restrict__ pm1, float* __restrict__ Y,
                                                          const int32_t* __restrict__ ids, const int* __restrict__ slots,
                                                          int32_t* __restrict__ slot_ids) {
  const int64_t per = wide / 8;
  for (int64_t e = blockIdx.x * static_cast<int64_t>(kBlock) + threadIdx.x; e < n_pad * per;
       e += static_cast<int64_t>(gridDim.x) * kBlock) {
    const int64_t row = e / per, c = (e - row * per) * 8;
    float x[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) x[q] = 0.f;
    if (row < n) {
      const float f = factor[row], g = pm1[row];
      if (slots && c == 0) slot_ids[row] = ids[row] >= 0 ? slots[ids[row]] : -1;
      float h[8], y[8];
      load_vec<GIST_STORE_BF16, 8>(H + row * ldh, c, h);
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        y[q] = h[q] * g;
        x[q] = f != 0.f ? h[q] * f : 0.f;
      }
      store_vec<8>(Y + row * wide + c, y);
    }
    store_as<GIST_STORE_BF16, 8>(F, row * wide + c, x);
  }
}

// Labelled rows, by a workgroup of 1,024; the result is thread 0's.  Four rows a load, four
// loads at a time: one workgroup reads a million labels in some 30 us.
__device__ __forceinline__ int count_labels(int64_t n, const int32_t* __restrict__ labels, const int32_t* __restrict__ n_dev,
                                            int (&sh)[16]) {
  int64_t real = n_dev ? max(0, *n_dev) : n;
  real = real < n ? real : n;
  int c = 0;
  const int64_t whole = real / 4;
#pragma unroll 4
  for (int64_t i = threadIdx.x; i < whole; i += 1024) {
    const intx4w v = *reinterpret_cast<const intx4w*>(labels + i * 4);
#pragma unroll
    for (int q = 0; q < 4; ++q) c += v[q] >= 0;
  }
  for (int64_t i = whole * 4 + threadIdx.x; i < real; i += 1024) c += labels[i] >= 0;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) c += __shfl_xor(c, o, 64);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = c;
  __syncthreads();
  c = 0;
  for (int w = 0; w < 16; ++w) c += sh[w];
  return c;
}

// What comes before a piece's products, each by workgroups of its own in one launch (a launch is
// some 3 us, which small problems consist of): the rows' first references scale <h, t_y>, 16 bytes a
// lane of as many lanes as a row has of them (8 to 64), and cleared marks of far rows; no class has a slot yet; and the gradients'
// factor.  `slots`, `factor`: or NULL.
struct Begin {
  int64_t row0, n, C, total;   // total: rows of all pieces
  int wide, lanes;
  float scale, gscale;
  const char* H;
  const char* T;
  int64_t ldh, ldt;
  const int32_t* labels;       // the piece's
  const int32_t* all_labels;
  const int32_t* n_dev;
  float* ref;
  int* far;
  int* slots;
  float* factor;
  int64_t ref_blocks, slot_blocks;
};
constexpr int kBegin = 1024;
__global__ __launch_bounds__(kBegin) void begin_kernel(Begin a) {
  __shared__ int sh[16];
  int64_t b = blockIdx.x;
  if (b >= a.ref_blocks + a.slot_blocks) {
    const int c = count_labels(a.total, a.all_labels, a.n_dev, sh);
    if (threadIdx.x == 0) *a.factor = c > 0 ? a.gscale / static_cast<float>(c) : 0.f;
    return;
  }
  if (b >= a.ref_blocks) {
    const int64_t c = (b - a.ref_blocks) * kBegin + threadIdx.x;
    if (c < a.C) a.slots[c] = kNoSlot;
    return;
  }
  const int lane = threadIdx.x & (a.lanes - 1);
  const int64_t row = (b * kBegin + threadIdx.x) / a.lanes;
  if (row >= a.n) return;                          // all of a row's lanes
  if (row % 256 == 0 && lane == 0) a.far[row / 256] = 0;
  const int y = !a.n_dev || a.row0 + row < *a.n_dev ? a.labels[row] : -1;
  float s = 0.f;
  if (y >= 0 && y < a.C) {
    for (int c = lane * 8; c < a.wide; c += a.lanes * 8) {
      float h[8], t[8];
      load_vec<GIST_STORE_BF16, 8>(a.H + row * a.ldh, c, h);
      load_vec<GIST_STORE_BF16, 8>(a.T + y * a.ldt, c, t);
#pragma unroll
      for (int q = 0; q < 8; ++q) s = fmaf(h[q], t[q], s);
    }
  }
  for (int o = a.lanes >> 1; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  s *= a.scale;
  // a reference that is no number, or none to speak of, would spoil rows whose other logits are; 0 may then lie far
  // above a row's largest logit, which makes it far as well
  if (lane == 0) a.ref[row] = fabsf(s) < 1e30f ? s : 0.f;
}

// Loss and the gradients' factor, in a fixed order: every workgroup a share of the rows, every
// thread a stride of it.  One workgroup gives the results; several leave theirs in `parts`, and a
// second launch of one joins them (200,000 rows by one workgroup: 30 us).
constexpr int64_t kLossRows = 16384;   // of a workgroup
constexpr int kLossParts = 256;        // at most
struct LossPart {
  double sum;
  int64_t count;
};
__global__ __launch_bounds__(1024) void loss_kernel(int64_t n, const float* __restrict__ logp,
                                                    const int32_t* __restrict__ labels, const int32_t* __restrict__ n_dev,
                                                    float gscale, int64_t share, LossPart* __restrict__ parts, int joined,
                                                    float* __restrict__ loss, float* __restrict__ factor) {
  __shared__ double sh[16];
  __shared__ int64_t sc[16];
  double s = 0.0;
  int64_t c = 0;
  if (joined > 0) {      // parts of the launch before
    if (threadIdx.x < joined) {
      s = parts[threadIdx.x].sum;
      c = parts[threadIdx.x].count;
    }
  } else {
    int64_t real = n_dev ? max(0, *n_dev) : n;
    real = real < n ? real : n;
    const int64_t first = blockIdx.x * share, last = min(real, first + share);   // share: a multiple of 4
    const int64_t whole = first + max(int64_t{0}, last - first) / 4 * 4;
#pragma unroll 4
    for (int64_t i = first + threadIdx.x * 4; i < whole; i += 4096) {   // as count_labels reads
      const floatx4 p = *reinterpret_cast<const floatx4*>(logp + i);
      const intx4w v = *reinterpret_cast<const intx4w*>(labels + i);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        s += p[q];
        c += v[q] >= 0;
      }
    }
    for (int64_t i = whole + threadIdx.x; i < last; i += 1024) {
      s += logp[i];
      c += labels[i] >= 0;
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    s += __shfl_xor(s, o, 64);
    c += __shfl_xor(c, o, 64);
  }
  if ((threadIdx.x & 63) == 0) {
    sh[threadIdx.x >> 6] = s;
    sc[threadIdx.x >> 6] = c;
  }
  __syncthreads();
  if (threadIdx.x != 0) return;
  s = 0.0;
  c = 0;
  for (int w = 0; w < 16; ++w) {
    s += sh[w];
    c += sc[w];
  }
  if (gridDim.x > 1) {
    parts[blockIdx.x] = LossPart{s, c};
    return;
  }
  *loss = c > 0 ? static_cast<float>(-s / c) : 0.f;
  if (factor) *factor = c > 0 ? gscale / static_cast<float>(c) : 0.f;
}

// out = f sum of the slices' partial results, in order; four elements a thread.  With factors of
// the rows: f (factor sum + pm1 T[ids]), 0 where the factor is.
struct Given {
  const float* row_factor;
  const float* pm1;
  const int32_t* ids;
  const char* T;
  int64_t ldt;
};
template <int STORE, int OPS>
__global__ __launch_bounds__(kBlock) void join_out_kernel(int64_t rows, int d, int64_t ldp, int slices, int64_t slice,
                                                          const float* __restrict__ part, const float* __restrict__ factor,
                                                          Given g, void* __restrict__ out, int64_t ldo) {
  const int per = static_cast<int>(ldp / 4);
  const float f = *factor;
  for (int64_t e = blockIdx.x * static_cast<int64_t>(kBlock) + threadIdx.x; e < rows * per;
       e += static_cast<int64_t>(gridDim.x) * kBlock) {
    const int64_t row = e / per;
    const int c = static_cast<int>(e - row * per) * 4;
    floatx4 v = *reinterpret_cast<const floatx4*>(part + row * ldp + c);
    for (int s = 1; s < slices; ++s) v += *reinterpret_cast<const floatx4*>(part + s * slice + row * ldp + c);
    if (g.row_factor) {
      const float rf = g.row_factor[row];
      const int id = g.ids[row];
      float t[4] = {};
      if (id >= 0) load4_16<OPS>(g.T + id * g.ldt, c, t);   // a row of T has a multiple of 64
      const float p = id >= 0 ? g.pm1[row] : 0.f;
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = rf == 0.f ? 0.f : fmaf(p, t[q], rf * v[q]);
    }
    if (c + 4 <= d && STORE != GIST_STORE_F32) {
      float x[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) x[q] = v[q] * f;
      int u[2];
      pack4<STORE == GIST_STORE_F32 ? static_cast<int>(GIST_STORE_BF16) : STORE>(x, u);
      typedef int intx2u __attribute__((ext_vector_type(2), aligned(2)));
      *reinterpret_cast<intx2u*>(static_cast<unsigned short*>(out) + row * ldo + c) = intx2u{u[0], u[1]};
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float x[1] = {v[q] * f};
        if (c + q < d) store_as<STORE, 1>(out, row * ldo + c + q, x);
      }
    }
  }
}

// fp32 pieces: a row's logits (a product's, not yet scaled) become its G, times the factor.  A row in the
// registers of THREADS threads, CH loads of four each: read once, written once.  200,000 rows of
// 41 classes, d 256, with gradients: 664 us by 256 threads a row and three reads (and one workgroup's loss), 370 so.
template <int THREADS, int CH>
__global__ __launch_bounds__(kBlock) void piece_kernel(int64_t row0, int64_t rows, int64_t n, int64_t C, float scale,
                                                       float* __restrict__ Z, int64_t ldz, const int32_t* __restrict__ labels,
                                                       const int32_t* __restrict__ n_dev, const float* __restrict__ factor,
                                                       int grad, float* __restrict__ lse_out, float* __restrict__ logp,
                                                       float* __restrict__ logp_out) {
  __shared__ float sm[kBlock / 64], ss[kBlock / 64];
  constexpr int RB = kBlock / THREADS;
  const int lane = threadIdx.x % THREADS;
  const int64_t real = n_dev ? max(0, *n_dev) : n;
  const float f = grad ? *factor : 0.f;
  for (int64_t i = blockIdx.x * static_cast<int64_t>(RB) + threadIdx.x / THREADS; i < rows;
       i += static_cast<int64_t>(gridDim.x) * RB) {
    float* const z = Z + i * ldz;
    const int64_t row = row0 + i;
    const int y = row < real ? labels[row] : -1;
    floatx4 v[CH];
    float m = -__builtin_inff();
#pragma unroll
    for (int h = 0; h < CH; ++h) {
      const int64_t c = (h * THREADS + lane) * 4;
      v[h] = floatx4{} - __builtin_inff();
      if (c < C) {     // ldz is a multiple of 4
        const floatx4 t = *reinterpret_cast<const floatx4*>(z + c);
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (c + q < C) v[h][q] = t[q] * scale;
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) m = fmaxf(m, v[h][q]);
    }
#pragma unroll
    for (int o = (THREADS < 64 ? THREADS : 64) / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
    if constexpr (THREADS > 64) {
      if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = m;
      __syncthreads();
      m = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3]));
    }
    const float ref = m == -__builtin_inff() ? 0.f : m;
    float s = 0.f;
#pragma unroll
    for (int h = 0; h < CH; ++h) {
      float p[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) p[q] = ex2((v[h][q] - ref) * kL);
      s += (p[0] + p[1]) + (p[2] + p[3]);
    }
#pragma unroll
    for (int o = (THREADS < 64 ? THREADS : 64) / 2; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    if constexpr (THREADS > 64) {
      if ((threadIdx.x & 63) == 0) ss[threadIdx.x >> 6] = s;
      __syncthreads();
      s = (ss[0] + ss[1]) + (ss[2] + ss[3]);
    }
    const float ls = lg2(s) * kLn2;
    if (lane == 0) {
      if (lse_out) lse_out[row] = m + ls;
      if (y < 0 || y >= C) {
        const float lp = y < 0 ? 0.f : __builtin_nanf("");
        logp[row] = lp;
        if (logp_out) logp_out[row] = lp;
      }
    }
    const float fs = y < 0 ? 0.f : f;
#pragma unroll
    for (int h = 0; h < CH; ++h) {
      const int64_t c = (h * THREADS + lane) * 4;
      floatx4 g;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float p = ex2((v[h][q] - m - ls) * kL);
        if (c + q == y && y < C) {
          const float lp = v[h][q] - m - ls;
          logp[row] = lp;
          if (logp_out) logp_out[row] = lp;
          p -= 1.f;
        }
        g[q] = y < 0 || c + q >= C ? 0.f : p * fs;
      }
      if (grad && c < ldz) *reinterpret_cast<floatx4*>(z + c) = g;
    }
  }
}

// The same for more than 2 kChunk classes: kChunk of them a workgroup, held in its registers, which leaves
// their maximum and sum for join_stats_kernel and the given class's logit; then G.  Whole
// calls with d = 64, loss alone, by piece_kernel and so: 1 row of 131,072 classes 82 and 28 us, 1,024
// rows 505 and 310 us; 1,024 rows of 9,000 classes 35 and 35 us; fewer classes are
// one or two chunks, and the joining launch is for nothing.
constexpr int kChunk = 4096;
__global__ __launch_bounds__(kBlock) void chunk_stats_kernel(int64_t row0, int64_t rows, int64_t n, int64_t C, float scale,
                                                             const float* __restrict__ Z, int64_t ldz,
                                                             const int32_t* __restrict__ labels, const int32_t* __restrict__ n_dev,
                                                             floatx2* __restrict__ stats, float* __restrict__ zy) {
  __shared__ float sm[kBlock / 64], ss[kBlock / 64];
  const int64_t i = blockIdx.y, c0 = static_cast<int64_t>(blockIdx.x) * kChunk, row = row0 + i;
  const float* const z = Z + i * ldz;
  constexpr int L = kChunk / (kBlock * 4);
  floatx4 v[L];
  float m = -__builtin_inff();
#pragma unroll
  for (int l = 0; l < L; ++l) {
    const int64_t c = c0 + (l * kBlock + threadIdx.x) * 4;
    v[l] = floatx4{} - __builtin_inff();
    if (c < C) {     // ldz is a multiple of 4
      const floatx4 t = *reinterpret_cast<const floatx4*>(z + c);
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (c + q < C) v[l][q] = t[q] * scale;
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) m = fmaxf(m, v[l][q]);
  }
  m = wave_max(m);
  if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = m;
  __syncthreads();
  m = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3]));
  const float ref = m == -__builtin_inff() ? 0.f : m;
  float s = 0.f;
#pragma unroll
  for (int l = 0; l < L; ++l)
#pragma unroll
    for (int q = 0; q < 4; ++q) s += ex2((v[l][q] - ref) * kL);
  s = wave_sum(s);
  if ((threadIdx.x & 63) == 0) ss[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x != 0) return;
  stats[blockIdx.x * rows + i] = floatx2{m, (ss[0] + ss[1]) + (ss[2] + ss[3])};
  const int64_t y = row < (n_dev ? static_cast<int64_t>(*n_dev) : n) ? labels[row] : -1;
  if (y >= c0 && y < min(C, c0 + kChunk)) zy[i] = z[y] * scale;
}
__global__ __launch_bounds__(kBlock) void chunk_grad_kernel(int64_t row0, int64_t n, int64_t C, float scale, float* __restrict__ Z,
                                                            int64_t ldz, const int32_t* __restrict__ labels,
                                                            const int32_t* __restrict__ n_dev, const float* __restrict__ factor,
                                                            const float* __restrict__ lse) {
  const int64_t i = blockIdx.y, c0 = static_cast<int64_t>(blockIdx.x) * kChunk, row = row0 + i;
  float* const z = Z + i * ldz;
  const int64_t y = row < (n_dev ? static_cast<int64_t>(*n_dev) : n) ? labels[row] : -1;
  const float f = *factor, l = lse[i];
#pragma unroll
  for (int h = 0; h < kChunk / (kBlock * 4); ++h) {
    const int64_t c = c0 + (h * kBlock + threadIdx.x) * 4;
    if (c >= ldz) break;
    floatx4 v = *reinterpret_cast<const floatx4*>(z + c);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      float p = ex2((v[q] * scale - l) * kL);
      if (c + q == y) p -= 1.f;
      v[q] = y < 0 || c + q >= C ? 0.f : p * f;
    }
    *reinterpret_cast<floatx4*>(z + c) = v;
  }
}

// The gradients' factor alone (fp32 pieces need it before their loss is known).
__global__ __launch_bounds__(1024) void count_kernel(int64_t n, const int32_t* __restrict__ labels,
                                                     const int32_t* __restrict__ n_dev, float gscale, float* __restrict__ factor) {
  __shared__ int sc[16];
  const int c = count_labels(n, labels, n_dev, sc);
  if (threadIdx.x == 0) *factor = c > 0 ? gscale / static_cast<float>(c) : 0.f;
}

// Rows of fp32 with those that are not labelled zeroed; four elements a thread.
__global__ __launch_bounds__(kBlock) void mask_rows_kernel(int64_t row0, int64_t rows, int64_t n, int d, const float* __restrict__ x,
                                                           int64_t ldx, float* __restrict__ y, const int32_t* __restrict__ labels,
                                                           const int32_t* __restrict__ n_dev) {
  const int64_t real = n_dev ? max(0, *n_dev) : n;
  const int per = (d + 3) / 4;
  for (int64_t e = blockIdx.x * static_cast<int64_t>(kBlock) + threadIdx.x; e < rows * per;
       e += static_cast<int64_t>(gridDim.x) * kBlock) {
    const int64_t i = e / per;
    const int c = static_cast<int>(e - i * per) * 4;
    float v[4] = {};
    if (row0 + i < real && labels[row0 + i] >= 0) load_some<GIST_STORE_F32, 4>(x, (row0 + i) * ldx + c, d - c, 0.f, v);
    store_some<GIST_STORE_F32, 4>(y, i * d + c, d - c, v);
  }
}

// ---- plans -----------------------------------------------------------------------------------

size_t up256(size_t x) { return (x + 255) & ~size_t{255}; }
int64_t up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }
unsigned grid_of(int64_t count) { return static_cast<unsigned>(std::max<int64_t>(1, std::min<int64_t>((count + kBlock - 1) / kBlock, 16384))); }

int size_of(int store) { return store == GIST_STORE_F32 ? 4 : store == GIST_STORE_E4M3 ? 1 : 2; }

// How a product is cut: tiles of 256 (one workgroup a CU) or 128 (two).
struct Cut {
  int tile;        // 256, 128, or 32 rows (a forward product of few rows)
  int tiles_m, tiles_n, slices, len;
};

// A gradient's product (M x N, `steps` of K).  A round of workgroups takes as long for one
// tile as for one on every CU, so K is cut where the tiles do not fill rounds: the
// number of slices with the least time in units of a whole product's tile, a
// fortieth of it added for every slice (its partial result is written and read).  Uncut, the call of 8,192
// rows, 50,001 classes, d 1,024 takes 2,996 us in place of 2,504, that of 1,024 rows, 50,000
// classes, d 2,048 1,271 in place of 807.  With room for 1 GiB of parts, so that dT is cut as
// well, these take 2,709 and 1,095.  Up to 256 slices in place of 64: 200,000 rows, 41 classes, d 256 446 us (452), in
// fp16 244 (257), 100,000 rows, 200 classes, d 128 202 (198); all others the same.  Tiles of 256 from a quarter of a round of them on (8,192 rows, 12,000
// classes, d 1,024: 719 us, 849 by tiles of 128).
Cut cut_of(int64_t M, int64_t N, int steps) {
  Cut c{};
  const int64_t t256 = ((M + 255) / 256) * ((N + 255) / 256);
  c.tile = t256 * 4 >= 256 && M >= 256 && N >= 256 ? 256 : 128;
  c.tiles_m = static_cast<int>((M + c.tile - 1) / c.tile);
  c.tiles_n = static_cast<int>((N + c.tile - 1) / c.tile);
  const int64_t tiles = static_cast<int64_t>(c.tiles_m) * c.tiles_n;
  const int64_t at_once = c.tile == 256 ? 256 : 512;
  const int64_t most_by_room = std::max<int64_t>(1, static_cast<int64_t>(kPartBytes / 4) / std::max<int64_t>(1, M * N));
  double best = 1e30;
  c.slices = 1;
  for (int s = 1; s <= 64 && s <= most_by_room && s * 4 <= std::max(4, steps); ++s) {
    const double t = static_cast<double>((tiles * s + at_once - 1) / at_once) / s + (s > 1 ? 0.025 * s : 0.0) *
                     static_cast<double>(tiles) / at_once;
    if (t < best * 0.999) {
      best = t;
      c.slices = s;
    }
  }
  c.len = (steps + c.slices - 1) / c.slices;
  c.slices = (steps + c.len - 1) / c.len;
  return c;
}

// The logits' product: rows of a tile by how many there are, and tiles of 256 from half a round of
// workgroups on.  In bf16, loss alone: 32 rows, 131,072 classes, d 1,024 62 us, 82 by tiles of 128; 1,024 rows,
// 12,000 classes (188 tiles of 256) 36 us and 41; with gradients 5,000 rows, 1,000 classes, d 64 (80 tiles)
// 91 us and 85.  (8-bit fragments are twice as large: a tile of 256 would not fit the
// registers.)
Cut cut_logits(int64_t C, int64_t n, int steps, bool eight) {
  Cut c{};
  if (n <= 32) c.tile = 32;
  else if (!eight && C > 128 && ((C + 255) / 256) * ((n + 255) / 256) >= 128) c.tile = 256;
  else c.tile = 128;
  const int bm = c.tile == 128 ? 128 : 256, bn = c.tile;
  c.tiles_m = static_cast<int>((C + bm - 1) / bm);
  c.tiles_n = static_cast<int>((n + bn - 1) / bn);
  c.slices = 1;
  c.len = steps;
  return c;
}

// Where everything lies in the workspace (offsets).
struct Plan {
  bool f32;                 // fp32 products
  int op;                   // store of the products' operands
  bool copy_h, copy_t;      // operands that the products cannot read where they are
  int64_t wide;             // elements of a row of both operands; fp32: of a piece's logits
  int64_t rows;             // forward, and fp32: rows of a piece
  int chunks;               // fp32 rows cut into so many parts (0: a workgroup a row)
  int64_t n_pad, Cp;        // rows of G or E; classes of a piece (a multiple of 256)
  Cut dh, dt;               // the gradients' products, of the first piece
  bool exps;                // rows piece by piece, by their exponentials
  bool parts_h;             // dH is summed in fp32 parts
  size_t h, hm, t, stats, zy, lse, logp, factor, loss_parts, g, ref, row_factor, far, pm1, ids, y, embed, slots,
      slot_ids, kept, part, z, gemm, total;
  size_t gemm_bytes;
};

// Rows that the products load as they are: whole 128-byte steps, 16-byte pieces, offsets within a
// tile of 32 bits.
bool direct(const void* p, int64_t ld, int d, int store) {
  const int e = size_of(store);
  return (static_cast<int64_t>(d) * e) % 128 == 0 && (ld * e) % 16 == 0 && aligned16(p) && ld <= (1 << 22);
}

constexpr int waves_m(int tile) { return tile == 32 ? 4 : 2; }

// `any`: room for operands at any address.
Plan plan_of(const gist_table_xent_desc* D, const void* H, const void* T, bool grad, bool any) {
  Plan p{};
  const int64_t n = D->n, C = D->C;
  const int d = D->d;
  p.f32 = D->store == GIST_STORE_F32 && D->dtype == GIST_DTYPE_F32;
  size_t o = 0;
  auto take = [&](size_t bytes) {
    const size_t at = o;
    o += up256(bytes);
    return at;
  };
  p.logp = take(static_cast<size_t>(n) * 4);
  p.factor = take(16);
  p.loss_parts = take(kLossParts * sizeof(LossPart));
  if (p.f32) {
    p.wide = up(C, 4);
    int64_t rows = static_cast<int64_t>(kPieceBytes / 4) / p.wide;
    rows = rows >= 256 ? rows / 256 * 256 : std::max<int64_t>(1, rows);
    p.rows = std::min(n, rows);
    p.z = take(static_cast<size_t>(p.rows) * p.wide * 4);
    p.chunks = C > 2 * kChunk ? static_cast<int>((C + kChunk - 1) / kChunk) : 0;
    if (p.chunks) {
      p.stats = take(static_cast<size_t>(p.rows) * p.chunks * 8);
      p.zy = take(static_cast<size_t>(p.rows) * 4);
      p.lse = take(static_cast<size_t>(p.rows) * 4);
    }
    if (grad) p.hm = take(static_cast<size_t>(p.rows) * d * 4);
    for (const int64_t r : {p.rows, n % p.rows}) {
      if (r == 0) continue;
      p.gemm_bytes = std::max(p.gemm_bytes, gemm_workspace(r, C, d, D->ldh, D->ldt, GIST_DTYPE_F32));
      if (!grad) continue;
      p.gemm_bytes = std::max(p.gemm_bytes, gemm_workspace(r, d, C, p.wide, D->ldt, GIST_DTYPE_F32));
      p.gemm_bytes = std::max(p.gemm_bytes, gemm_workspace(C, d, r, p.wide, d, GIST_DTYPE_F32));
    }
    p.gemm = take(p.gemm_bytes);
    p.total = o;
    return p;
  }
  p.op = D->store == GIST_STORE_F32 ? static_cast<int>(GIST_STORE_BF16) : D->store;
  const int e = size_of(p.op);
  p.wide = up(d, 128 / e);
  p.copy_h = D->store == GIST_STORE_F32 || !direct(H, D->ldh, d, D->store);
  p.copy_t = D->store == GIST_STORE_F32 || !direct(T, D->ldt, d, D->store);
  // at most so many rows at a time that their maxima and sums take a piece's room; every cut has
  // at most a part for 64 classes and one more tile
  const int64_t parts = C / 64 + 4;
  p.rows = std::min(n, std::max<int64_t>(256, static_cast<int64_t>(kPieceBytes / 8) / parts / 256 * 256));
  p.exps = grad && p.op == GIST_STORE_BF16;
  if (p.exps) p.rows = std::min(p.rows, std::max<int64_t>(256, static_cast<int64_t>(kExpBytes / 2) / up(C, 256) / 256 * 256));
  p.stats = take(static_cast<size_t>(parts) * p.rows * 8);
  p.zy = take(static_cast<size_t>(n) * 4);
  p.lse = take(static_cast<size_t>(n) * 4);
  if (p.copy_h || any) p.h = take(static_cast<size_t>(n) * p.wide * e);
  if (p.copy_t || any) p.t = take(static_cast<size_t>(C) * p.wide * e);
  if (p.exps) {
    const int64_t ldp = up(d, 4), rn = p.rows;
    p.n_pad = up(rn, 256);
    p.Cp = up(C, 256);
    p.hm = take(static_cast<size_t>(up(rn, 64)) * p.wide * 2);
    p.g = take(static_cast<size_t>(p.n_pad) * p.Cp * 2);
    p.ref = take(static_cast<size_t>(rn) * 4);
    p.row_factor = take(static_cast<size_t>(rn) * 4);
    p.far = take(static_cast<size_t>(p.n_pad / 256) * 4);
    p.dh = cut_of(d, rn, static_cast<int>(up(C, 64) / 64));
    p.dt = cut_of(d, C, static_cast<int>(up(rn, 64) / 64));
    p.parts_h = p.dh.slices > 1;
    const bool parts_t = p.dt.slices > 1 || rn < n;
    p.part = take((p.parts_h ? static_cast<size_t>(p.dh.slices) * rn * ldp * 4 : 0) +
                  (parts_t ? static_cast<size_t>(p.dt.slices) * C * ldp * 4 : 0));
    if (p.dt.slices == 1) {
      p.slots = take(static_cast<size_t>(C) * 4);
      p.slot_ids = take(static_cast<size_t>(rn) * 4);
      p.kept = take(static_cast<size_t>(rn) * ldp * 4);
    }
    p.pm1 = take(static_cast<size_t>(rn) * 4);
    p.ids = take(static_cast<size_t>(rn) * 4);
    p.y = take(static_cast<size_t>(rn) * p.wide * 4);
    p.embed = take(std::max(embed_grad_workspace(rn, C, d), embed_grad_workspace(rn, rn, d)));   // serves fewer ids
  } else if (grad) {
    p.n_pad = up(n, 256);
    const int64_t fit = static_cast<int64_t>(kPieceBytes / 2) / p.n_pad / 256 * 256;
    p.Cp = std::min(up(C, 256), std::max<int64_t>(256, fit));
    const int64_t cn = std::min(C, p.Cp), ldp = up(d, 4);
    p.hm = take(static_cast<size_t>(up(n, 64)) * p.wide * 2);
    p.g = take(static_cast<size_t>(p.n_pad) * p.Cp * 2);
    p.dh = cut_of(d, n, static_cast<int>(up(cn, 64) / 64));
    p.dt = cut_of(d, cn, static_cast<int>(up(n, 64) / 64));
    p.parts_h = p.dh.slices > 1 || p.Cp < C;
    size_t part = p.parts_h ? static_cast<size_t>(p.dh.slices) * n * ldp * 4 : 0;
    if (p.dt.slices > 1) part += static_cast<size_t>(p.dt.slices) * cn * ldp * 4;
    p.part = take(part);
  }
  p.total = o;
  return p;
}

template <int STORE, int EPI, bool PT, bool QT>
void launch_product(hipStream_t st, int tile, const Prod& a) {
  const dim3 grid(static_cast<unsigned>(static_cast<int64_t>(a.tiles_m) * a.tiles_n * a.slices));
  if constexpr (EPI != kPart && EPI != kOut) {
    if (tile == 32) {
      hipLaunchKernelGGL((product_kernel<STORE, 4, 2, 4, 1, 4, PT, QT, EPI>), grid, dim3(256), 0, st, a);
      return;
    }
  }
  if constexpr (STORE != GIST_STORE_E4M3) {
    if (tile == 256) {
      hipLaunchKernelGGL((product_kernel<STORE, 8, 4, 2, 4, 2, PT, QT, EPI>), grid, dim3(512), 0, st, a);
      return;
    }
  }
  hipLaunchKernelGGL((product_kernel<STORE, 4, 4, 2, 2, 2, PT, QT, EPI>), grid, dim3(256), 0, st, a);
}

void set_cut(Prod& a, const Cut& c) {
  a.tiles_m = c.tiles_m;
  a.tiles_n = c.tiles_n;
  a.slices = c.slices;
  a.len = c.len;
}

template <int STORE>
void join_out(hipStream_t st, const gist_table_xent_desc* D, int64_t rows, int slices, int64_t slice, const float* part,
              const float* factor, const Given& g, void* out, int64_t ldo) {
  const int64_t ldp = up(D->d, 4);
  const dim3 grid(grid_of(rows * ldp / 4));
  if (D->store == GIST_STORE_F32)
    hipLaunchKernelGGL((join_out_kernel<GIST_STORE_F32, STORE>), grid, dim3(kBlock), 0, st, rows, D->d, ldp, slices, slice, part,
                       factor, g, out, ldo);
  else
    hipLaunchKernelGGL((join_out_kernel<STORE, STORE>), grid, dim3(kBlock), 0, st, rows, D->d, ldp, slices, slice, part, factor,
                       g, out, ldo);
}

template <int SRC, int DST>
void copy_rows(hipStream_t st, int64_t n, int64_t n_pad, int d, int64_t wide, const void* x, int64_t ldx, void* y,
               const int32_t* labels, const int32_t* n_dev) {
  ProfScope ps(st, "table_xent_copy", 0.0, static_cast<double>(n_pad) * wide * (size_of(SRC) + size_of(DST)));
  hipLaunchKernelGGL((copy_rows_kernel<SRC, DST>), dim3(grid_of(n_pad * wide / 8)), dim3(kBlock), 0, st, n, n_pad, d,
                     static_cast<int>(wide), x, ldx, y, labels, n_dev);
}

gist_status run_loss(hipStream_t st, int64_t n, const float* logp, const int32_t* labels, const int32_t* n_dev, float gscale,
                     LossPart* parts, float* loss, float* factor) {
  ProfScope ps(st, "table_xent_loss", 0.0, 8.0 * n);
  const int64_t share = std::max(kLossRows, up((n + kLossParts - 1) / kLossParts, 4));
  const int blocks = static_cast<int>((n + share - 1) / share);
  hipLaunchKernelGGL(loss_kernel, dim3(static_cast<unsigned>(blocks)), dim3(1024), 0, st, n, logp, labels, n_dev, gscale, share,
                     parts, 0, loss, factor);
  if (blocks > 1)
    hipLaunchKernelGGL(loss_kernel, dim3(1), dim3(1024), 0, st, n, logp, labels, n_dev, gscale, share, parts, blocks, loss,
                       factor);
  return check_launch("table_xent_loss");
}

// The same cut for fewer rows (N).
Cut cut_rows(Cut c, int64_t N) {
  c.tiles_n = static_cast<int>((N + c.tile - 1) / c.tile);
  return c;
}

// Operands of 16 or 8 bits, ready to be loaded: H and T with ldh and ldt bytes from row to row.
template <int STORE>
gist_status run16(hipStream_t st, const gist_table_xent_desc* D, const Plan& p, const char* H, int64_t ldh, const char* T,
                  int64_t ldt, const float* h_scale, const float* t_scale, const int32_t* labels, const int32_t* n_dev,
                  float* loss, float* logp, float* lse, void* dH, void* dT, char* w) {
  const int64_t n = D->n, C = D->C;
  const int d = D->d, e = size_of(STORE);
  const bool grad = dH != nullptr;
  auto f32 = [&](size_t at) { return reinterpret_cast<float*>(w + at); };
  Prod a{};
  a.P = T;
  a.ldp = ldt;
  a.ldq = ldh;
  a.M = a.RP = C;
  a.steps = static_cast<int>(p.wide * e / 128);
  a.scale = D->scale;
  a.ps = t_scale;
  a.stats = reinterpret_cast<floatx2*>(w + p.stats);
  float* const ref = p.exps ? f32(p.ref) : nullptr;
  float* const row_factor = p.exps ? f32(p.row_factor) : nullptr;
  int* const far = p.exps ? reinterpret_cast<int*>(w + p.far) : nullptr;
  float* const pm1 = p.exps ? f32(p.pm1) : nullptr;
  int32_t* const ids = p.exps ? reinterpret_cast<int32_t*>(w + p.ids) : nullptr;
  a.lse = ref;
  a.out = w + p.g;
  a.ldo = p.Cp;
  a.far = far;
  for (int64_t r0 = 0; r0 < n; r0 += p.rows) {
    const int64_t rn = std::min(p.rows, n - r0);
    const Cut c = cut_logits(C, rn, a.steps, STORE == GIST_STORE_E4M3);
    set_cut(a, c);
    a.Q = H + r0 * ldh;
    a.N = a.RQ = a.ldstat = rn;
    a.row0 = r0;
    a.n_dev = n_dev;
    a.qs = h_scale ? h_scale + r0 : nullptr;
    a.labels = labels + r0;
    a.zy = f32(p.zy) + r0;
    // The last piece's product writes dT where it is not cut; before, and where it is, parts are kept.
    const bool straight = p.exps && p.dt.slices == 1 && r0 + rn == n;
    int* const slots = straight ? reinterpret_cast<int*>(w + p.slots) : nullptr;
    int32_t* const slot_ids = straight ? reinterpret_cast<int32_t*>(w + p.slot_ids) : nullptr;
    if constexpr (STORE == GIST_STORE_BF16) {
      if (p.exps) {
        Begin b{};
        b.row0 = r0;
        b.n = rn;
        b.C = C;
        b.total = n;
        b.wide = static_cast<int>(p.wide);
        b.scale = D->scale;
        b.gscale = D->grad_scale * D->scale;
        b.H = a.Q;
        b.T = T;
        b.ldh = ldh;
        b.ldt = ldt;
        b.labels = a.labels;
        b.all_labels = labels;
        b.n_dev = n_dev;
        b.ref = ref;
        b.far = far;
        b.slots = slots;
        b.factor = f32(p.factor);
        b.lanes = 8;
        while (b.lanes < 64 && b.lanes * 8 < b.wide) b.lanes *= 2;
        b.ref_blocks = (rn * b.lanes + kBegin - 1) / kBegin;
        b.slot_blocks = straight ? (C + kBegin - 1) / kBegin : 0;
        ProfScope ps(st, "table_xent_begin", 0.0, 4.0 * rn * d);
        hipLaunchKernelGGL(begin_kernel, dim3(static_cast<unsigned>(b.ref_blocks + b.slot_blocks + (r0 == 0))), dim3(kBegin), 0,
                           st, b);
        GIST_LAUNCHED("table_xent_begin");
      }
    }
    {
      ProfScope ps(st, "table_xent_logits", 2.0 * rn * C * d,
                   static_cast<double>(rn + C) * d * e + (p.exps ? 2.0 * rn * C : 0.0));
      if constexpr (STORE == GIST_STORE_BF16) {
        if (p.exps) launch_product<STORE, kExp, false, false>(st, c.tile, a);
        else launch_product<STORE, kStats, false, false>(st, c.tile, a);
      } else {
        launch_product<STORE, kStats, false, false>(st, c.tile, a);
      }
      GIST_LAUNCHED("table_xent_logits");
    }
    {
      const int parts = c.tiles_m * waves_m(c.tile);
      ProfScope ps(st, "table_xent_join", 0.0, 8.0 * parts * rn);
      // few parts leave most threads of a workgroup of few rows without one (200,000 rows of 2 parts
      // by 32 rows a workgroup: 29 us)
      auto launch = [&](auto kernel, int64_t per) {
        hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>((rn + per - 1) / per)), dim3(1024), 0, st, r0, rn, C, parts, a.stats,
                           rn, a.zy, a.labels, n_dev, f32(p.lse) + r0, lse ? lse + r0 : nullptr, f32(p.logp) + r0,
                           logp ? logp + r0 : nullptr, ref, row_factor, far);
      };
      if (rn <= 256) launch(join_stats_kernel<4>, 4);
      else if (parts <= 8) launch(join_stats_kernel<256>, 256);
      else launch(join_stats_kernel<32>, 32);
      GIST_LAUNCHED("table_xent_join");
    }
    if constexpr (STORE == GIST_STORE_BF16) {
      if (!p.exps) continue;
      {
        ProfScope ps(st, "table_xent_again", 0.0, 0.0);   // does nothing but for far rows
        launch_product<STORE, kAgain, false, false>(st, c.tile, a);
        GIST_LAUNCHED("table_xent_again");
      }
      {
        ProfScope ps(st, "table_xent_given", 0.0, 18.0 * rn);
        hipLaunchKernelGGL(given_kernel, dim3(static_cast<unsigned>((rn + kBlock - 1) / kBlock)), dim3(kBlock), 0, st, r0, rn, C,
                           f32(p.logp) + r0, a.labels, n_dev, reinterpret_cast<unsigned short*>(w + p.g), p.Cp, pm1, ids,
                           slots);
        GIST_LAUNCHED("table_xent_given");
      }
      float* const Y = f32(p.y);
      {
        ProfScope ps(st, "table_xent_factored", 0.0, 8.0 * rn * d);
        hipLaunchKernelGGL(factored_kernel, dim3(grid_of(up(rn, 64) * p.wide / 8)), dim3(kBlock), 0, st, rn, up(rn, 64), p.wide,
                           a.Q, ldh, row_factor, w + p.hm, pm1, Y, ids, slots, slot_ids);
        GIST_LAUNCHED("table_xent_factored");
      }
      const int64_t ldp = up(d, 4), moved = 2 * rn * C;
      float* const part_h = f32(p.part);
      float* const part_t = part_h + (p.parts_h ? p.dh.slices * p.rows * ldp : 0);
      {   // dH [rn][d] = E T, a row times its factor.  E is zero behind the last class.
        Prod b{};
        b.P = T;
        b.ldp = ldt;
        b.Q = w + p.g;
        b.ldq = p.Cp * 2;
        b.M = d;
        b.N = b.RQ = rn;
        b.RP = p.wide;
        b.KP = C;
        b.steps = static_cast<int>(up(C, 64) / 64);
        const Cut k = rn == p.rows ? p.dh : cut_rows(p.dh, rn);
        set_cut(b, k);
        char* const out = static_cast<char*>(dH) + r0 * D->lddh * size_of(D->store);
        ProfScope ps(st, "table_xent_dh", 2.0 * rn * C * d, moved + static_cast<double>(rn + C) * d * e);
        if (p.parts_h) {
          b.out = part_h;
          b.ldo = ldp;
          launch_product<STORE, kPart, true, false>(st, k.tile, b);
          GIST_LAUNCHED("table_xent_dh");
          join_out<STORE>(st, D, rn, b.slices, rn * ldp, part_h, f32(p.factor), Given{row_factor, pm1, ids, T, ldt}, out,
                          D->lddh);
        } else {
          b.out = out;
          b.ldo = D->lddh;
          b.factor = f32(p.factor);
          b.row_factor = row_factor;
          b.pm1 = pm1;
          b.ids = ids;
          b.T = T;
          b.ldt = ldt;
          b.out_store = D->store;
          launch_product<STORE, kOut, true, false>(st, k.tile, b);
        }
        GIST_LAUNCHED("table_xent_dh");
      }
      {   // dT [C][d] (+)= E^T H, over the piece's rows
        Prod b{};
        b.P = w + p.hm;
        b.ldp = p.wide * 2;
        b.Q = w + p.g;
        b.ldq = p.Cp * 2;
        b.M = d;
        b.N = C;
        b.RP = p.wide;
        b.RQ = up(C, c.tile == 128 ? 128 : 256);    // columns of E that have been written
        b.KP = up(rn, 64);
        b.KQ = std::min(b.KP, up(rn, c.tile));      // and rows
        b.steps = static_cast<int>(b.KP / 64);
        set_cut(b, p.dt);
        b.len = (b.steps + b.slices - 1) / b.slices;
        b.slices = (b.steps + b.len - 1) / b.len;   // no more than the first piece's
        ProfScope ps(st, "table_xent_dt", 2.0 * rn * C * d, moved + static_cast<double>(rn + C) * d * e);
        if (straight) {
          b.out = dT;
          b.ldo = D->lddt;
          b.factor = f32(p.factor);
          b.out_store = D->store;
          b.slots = slots;
          b.rows = f32(p.kept);
          b.part = r0 > 0 ? part_t : nullptr;
          b.ldr = ldp;
          launch_product<STORE, kOut, true, true>(st, p.dt.tile, b);
        } else {
          b.out = part_t;
          b.ldo = ldp;
          b.add = r0 > 0;
          launch_product<STORE, kPart, true, true>(st, p.dt.tile, b);
        }
        GIST_LAUNCHED("table_xent_dt");
      }
      {   // and the given classes' rows
        const gist_status s =
            straight ? embed_grad(st, rn, p.rows, d, slot_ids, 1.f, Y, p.wide, true, -1.f, f32(p.kept), ldp, w + p.embed)
                     : embed_grad(st, rn, C, d, ids, 1.f, Y, p.wide, true, -1.f, part_t, ldp, w + p.embed);
        if (s != GIST_OK) return s;
      }
      if (straight) {
        ProfScope ps(st, "table_xent_given_out", 0.0, 6.0 * rn * d);
        const dim3 grid(static_cast<unsigned>(rn));
        if (D->store == GIST_STORE_F32)
          hipLaunchKernelGGL(given_out_kernel<GIST_STORE_F32>, grid, dim3(kBlock), 0, st, rn, d, ids, slot_ids, f32(p.kept), ldp,
                             f32(p.factor), dT, D->lddt);
        else
          hipLaunchKernelGGL(given_out_kernel<STORE>, grid, dim3(kBlock), 0, st, rn, d, ids, slot_ids, f32(p.kept), ldp,
                             f32(p.factor), dT, D->lddt);
        GIST_LAUNCHED("table_xent_given_out");
      } else if (r0 + rn == n) {
        ProfScope ps(st, "table_xent_dt_join", 0.0, 4.0 * p.dt.slices * C * ldp);
        join_out<STORE>(st, D, C, p.dt.slices, C * ldp, part_t, f32(p.factor), Given{}, dT, D->lddt);
        GIST_LAUNCHED("table_xent_dt_join");
      }
    }
  }
  constexpr float kUnhold = STORE == GIST_STORE_F16 ? 1.f / 32768.f : 1.f;
  const gist_status sl = run_loss(st, n, f32(p.logp), labels, n_dev, D->grad_scale * D->scale * kUnhold,
                                  reinterpret_cast<LossPart*>(w + p.loss_parts), loss, grad && !p.exps ? f32(p.factor) : nullptr);
  if (sl != GIST_OK) return sl;
  if (!grad || p.exps) return GIST_OK;
  if constexpr (STORE == GIST_STORE_F16) {
    const int64_t ldp = up(d, 4);
    char* const hm = w + p.hm;
    char* const g = w + p.g;
    float* const factor = f32(p.factor);
    float* const part_h = f32(p.part);
    float* const part_t = part_h + (p.parts_h ? p.dh.slices * n * ldp : 0);
    a.Q = H;
    a.N = a.RQ = n;
    a.labels = labels;
    a.row0 = 0;
    a.lse = f32(p.lse);
    for (int64_t c0 = 0; c0 < C; c0 += p.Cp) {
      const int64_t cn = std::min(p.Cp, C - c0);
      const int64_t moved = 2 * n * cn;
      const char* const Tp = T + c0 * ldt;
      const Cut cg = cut_logits(cn, n, a.steps, false);
      {   // G [n_pad][Cp]: all rows and classes of the tiles
        Prod b = a;
        set_cut(b, cg);
        b.P = Tp;
        b.M = b.RP = cn;
        b.class0 = c0;
        b.out = g;
        b.ldo = p.Cp;
        ProfScope ps(st, "table_xent_grad", 2.0 * n * cn * d, static_cast<double>(n + cn) * d * e + moved);
        launch_product<STORE, kGrad, false, false>(st, cg.tile, b);
        GIST_LAUNCHED("table_xent_grad");
      }
      {   // dH [n][d]: G T over the piece's classes.  G is zero behind the last class.
        Prod b{};
        b.P = Tp;
        b.ldp = ldt;
        b.Q = g;
        b.ldq = p.Cp * 2;
        b.M = d;
        b.N = b.RQ = n;
        b.RP = p.wide;
        b.KP = cn;
        b.steps = static_cast<int>(up(cn, 64) / 64);
        set_cut(b, p.dh);
        b.len = (b.steps + b.slices - 1) / b.slices;
        b.slices = (b.steps + b.len - 1) / b.len;   // no more than the first piece's
        ProfScope ps(st, "table_xent_dh", 2.0 * n * cn * d, moved + static_cast<double>(n + cn) * d * e);
        if (p.parts_h) {
          b.out = part_h;
          b.ldo = ldp;
          b.add = c0 > 0;
          launch_product<STORE, kPart, true, false>(st, p.dh.tile, b);
        } else {
          b.out = dH;
          b.ldo = D->lddh;
          b.factor = factor;
          b.out_store = D->store;
          launch_product<STORE, kOut, true, false>(st, p.dh.tile, b);
        }
        GIST_LAUNCHED("table_xent_dh");
      }
      {   // dT [cn][d]: G^T H over the rows.  The copy of H is zero behind the last row.
        Prod b{};
        b.P = hm;
        b.ldp = p.wide * 2;
        b.Q = g;
        b.ldq = p.Cp * 2;
        b.M = d;
        b.N = cn;
        b.RP = p.wide;
        b.RQ = up(cn, cg.tile == 128 ? 128 : 256);   // columns of G that have been written
        b.KP = up(n, 64);
        b.KQ = std::min(b.KP, up(n, cg.tile));       // and rows
        b.steps = static_cast<int>(b.KP / 64);
        set_cut(b, p.dt);
        b.tiles_n = static_cast<int>((cn + p.dt.tile - 1) / p.dt.tile);
        char* const out = static_cast<char*>(dT) + c0 * D->lddt * size_of(D->store);
        ProfScope ps(st, "table_xent_dt", 2.0 * n * cn * d, moved + static_cast<double>(n + cn) * d * e);
        if (p.dt.slices > 1) {
          b.out = part_t;
          b.ldo = ldp;
          launch_product<STORE, kPart, true, true>(st, p.dt.tile, b);
          GIST_LAUNCHED("table_xent_dt");
          join_out<STORE>(st, D, cn, b.slices, cn * ldp, part_t, factor, Given{}, out, D->lddt);
        } else {
          b.out = out;
          b.ldo = D->lddt;
          b.factor = factor;
          b.out_store = D->store;
          launch_product<STORE, kOut, true, true>(st, p.dt.tile, b);
        }
        GIST_LAUNCHED("table_xent_dt");
      }
    }
    if (p.parts_h) {
      ProfScope ps(st, "table_xent_dh_join", 0.0, 4.0 * p.dh.slices * n * ldp);
      join_out<STORE>(st, D, n, p.dh.slices, n * ldp, part_h, factor, Given{}, dH, D->lddh);
      GIST_LAUNCHED("table_xent_dh_join");
    }
  }
  return GIST_OK;
}

template <int SRC, int STORE>
gist_status run_copied(hipStream_t st, const gist_table_xent_desc* D, const Plan& p, const void* H, const float* h_scale,
                       const void* T, const float* t_scale, const int32_t* labels, const int32_t* n_dev, float* loss,
                       float* logp, float* lse, void* dH, void* dT, char* w) {
  const int e = size_of(STORE);
  const char* h = static_cast<const char*>(H);
  const char* t = static_cast<const char*>(T);
  int64_t ldh = D->ldh * e, ldt = D->ldt * e;
  if (p.copy_h) {
    copy_rows<SRC, STORE>(st, D->n, D->n, D->d, p.wide, H, D->ldh, w + p.h, nullptr, nullptr);
    h = w + p.h;
    ldh = p.wide * e;
  }
  if (p.copy_t) {
    copy_rows<SRC, STORE>(st, D->C, D->C, D->d, p.wide, T, D->ldt, w + p.t, nullptr, nullptr);
    t = w + p.t;
    ldt = p.wide * e;
  }
  if constexpr (STORE == GIST_STORE_F16)
    if (dH) copy_rows<SRC, STORE>(st, D->n, up(D->n, 64), D->d, p.wide, H, D->ldh, w + p.hm, labels, n_dev);
  GIST_LAUNCHED("table_xent_copy");
  return run16<STORE>(st, D, p, h, ldh, t, ldt, h_scale, t_scale, labels, n_dev, loss, logp, lse, dH, dT, w);
}

gist_status run32(hipStream_t st, const gist_table_xent_desc* D, const Plan& p, const float* H, const float* T,
                  const int32_t* labels, const int32_t* n_dev, float* loss, float* logp, float* lse, float* dH, float* dT,
                  char* w) {
  const int64_t n = D->n, C = D->C;
  const int d = D->d;
  const bool grad = dH != nullptr;
  float* const z = reinterpret_cast<float*>(w + p.z);
  float* const hm = reinterpret_cast<float*>(w + p.hm);
  float* const logp_ws = reinterpret_cast<float*>(w + p.logp);
  float* const factor = reinterpret_cast<float*>(w + p.factor);
  void* const gws = w + p.gemm;
  if (grad) {
    ProfScope ps(st, "table_xent_count", 0.0, 4.0 * n);
    hipLaunchKernelGGL(count_kernel, dim3(1), dim3(1024), 0, st, n, labels, n_dev, D->grad_scale * D->scale, factor);
    GIST_LAUNCHED("table_xent_count");
  }
  for (int64_t r0 = 0; r0 < n; r0 += p.rows) {
    const int64_t rn = std::min(p.rows, n - r0);
    Operand A, B;
    GemmOut O;
    A.p0 = H + r0 * D->ldh;
    A.ld0 = D->ldh;
    B.p0 = T;
    B.ld0 = D->ldt;
    O.c0 = z;
    O.ldc0 = p.wide;
    gist_status s = gemm(st, rn, C, d, A, B, O, GIST_DTYPE_F32, gws, p.gemm_bytes);
    if (s != GIST_OK) return s;
    if (p.chunks) {
      float* const zy = reinterpret_cast<float*>(w + p.zy);
      float* const l = reinterpret_cast<float*>(w + p.lse);
      floatx2* const stats = reinterpret_cast<floatx2*>(w + p.stats);
      const dim3 grid(static_cast<unsigned>(p.chunks), static_cast<unsigned>(rn));
      ProfScope ps(st, "table_xent_chunks", 0.0, (grad ? 12.0 : 4.0) * rn * C);
      hipLaunchKernelGGL(chunk_stats_kernel, grid, dim3(kBlock), 0, st, r0, rn, n, C, D->scale, z, p.wide, labels, n_dev, stats,
                         zy);
      GIST_LAUNCHED("table_xent_chunks");
      hipLaunchKernelGGL(join_stats_kernel<4>, dim3(static_cast<unsigned>((rn + 3) / 4)), dim3(1024), 0, st, r0, rn, C, p.chunks,
                         stats, rn, zy, labels + r0, n_dev, l, lse ? lse + r0 : nullptr, logp_ws + r0, logp ? logp + r0 : nullptr,
                         nullptr, nullptr, nullptr);
      GIST_LAUNCHED("table_xent_chunks");
      if (grad) {
        hipLaunchKernelGGL(chunk_grad_kernel, grid, dim3(kBlock), 0, st, r0, n, C, D->scale, z, p.wide, labels, n_dev, factor, l);
        GIST_LAUNCHED("table_xent_chunks");
      }
    } else {
      ProfScope ps(st, "table_xent_piece", 0.0, (grad ? 8.0 : 4.0) * rn * C);
      auto launch = [&](auto kernel, int threads) {
        const int64_t g = std::min<int64_t>((rn * threads + kBlock - 1) / kBlock, 1 << 20);
        hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(g)), dim3(kBlock), 0, st, r0, rn, n, C, D->scale, z, p.wide, labels,
                           n_dev, factor, grad ? 1 : 0, lse, logp_ws, logp);
      };
      if (C <= 64) launch(piece_kernel<16, 1>, 16);
      else if (C <= 256) launch(piece_kernel<64, 1>, 64);
      else if (C <= 1024) launch(piece_kernel<64, 4>, 64);
      else launch(piece_kernel<kBlock, 2 * kChunk / (4 * kBlock)>, kBlock);
      GIST_LAUNCHED("table_xent_piece");
    }
    if (!grad) continue;
    {
      ProfScope ps(st, "table_xent_mask", 0.0, 8.0 * rn * d);
      hipLaunchKernelGGL(mask_rows_kernel, dim3(grid_of(rn * ((d + 3) / 4))), dim3(kBlock), 0, st, r0, rn, n, d, H, D->ldh, hm, labels, n_dev);
      GIST_LAUNCHED("table_xent_mask");
    }
    // dH = G T: T's rows are values of K
    Operand G1, T1;
    GemmOut O1;
    G1.p0 = z;
    G1.ld0 = p.wide;
    T1.p0 = T;
    T1.ld0 = D->ldt;
    T1.k_major = false;
    O1.c0 = dH + r0 * D->lddh;
    O1.ldc0 = D->lddh;
    s = gemm(st, rn, d, C, G1, T1, O1, GIST_DTYPE_F32, gws, p.gemm_bytes);
    if (s != GIST_OK) return s;
    // dT += G^T H: both operands' rows are values of K
    Operand G2, H2;
    GemmOut O2;
    G2.p0 = z;
    G2.ld0 = p.wide;
    G2.k_major = false;
    H2.p0 = hm;
    H2.ld0 = d;
    H2.k_major = false;
    O2.c0 = dT;
    O2.ldc0 = D->lddt;
    O2.sgd = r0 > 0;     // pieces after the first add to it: C <- C - (-1) product
    O2.lr = -1.f;
    s = gemm(st, C, d, rn, G2, H2, O2, GIST_DTYPE_F32, gws, p.gemm_bytes);
    if (s != GIST_OK) return s;
  }
  return run_loss(st, n, logp_ws, labels, n_dev, 0.f, reinterpret_cast<LossPart*>(w + p.loss_parts), loss, nullptr);
}

__global__ __launch_bounds__(kBlock) void zero_rows_kernel(int64_t rows, int64_t bytes, char* __restrict__ x, int64_t ld) {
  for (int64_t e = blockIdx.x * static_cast<int64_t>(kBlock) + threadIdx.x; e < rows * bytes;
       e += static_cast<int64_t>(gridDim.x) * kBlock)
    x[e / bytes * ld + e % bytes] = 0;
}

}  // namespace

size_t table_xent_workspace(const gist_table_xent_desc* D, bool grad) {
  return D->n == 0 ? 0 : plan_of(D, nullptr, nullptr, grad, true).total;
}

size_t table_xent_need(const gist_table_xent_desc* D, const void* H, const void* T, bool grad) {
  return D->n == 0 ? 0 : plan_of(D, H, T, grad, false).total;
}

gist_status table_xent(hipStream_t st, const gist_table_xent_desc* D, const void* H, const float* h_scale, const void* T,
                       const float* t_scale, const int32_t* labels, const int32_t* n_dev, float* loss, float* logp,
                       float* lse, void* dH, void* dT, void* ws) {
  char* const w = static_cast<char*>(ws);
  if (D->n == 0) {
    if (dT) {
      const int64_t bytes = static_cast<int64_t>(D->d) * size_of(D->store);
      hipLaunchKernelGGL(zero_rows_kernel, dim3(grid_of(D->C * bytes)), dim3(kBlock), 0, st, D->C, bytes,
                         static_cast<char*>(dT), D->lddt * size_of(D->store));
    }
    return fill_zero(st, loss, 1);
  }
  const Plan p = plan_of(D, H, T, dH != nullptr, false);
  if (p.f32)
    return run32(st, D, p, static_cast<const float*>(H), static_cast<const float*>(T), labels, n_dev, loss, logp, lse,
                 static_cast<float*>(dH), static_cast<float*>(dT), w);
  switch (D->store) {
    case GIST_STORE_F32:
      return run_copied<GIST_STORE_F32, GIST_STORE_BF16>(st, D, p, H, nullptr, T, nullptr, labels, n_dev, loss, logp, lse, dH, dT, w);
    case GIST_STORE_BF16:
      return run_copied<GIST_STORE_BF16, GIST_STORE_BF16>(st, D, p, H, nullptr, T, nullptr, labels, n_dev, loss, logp, lse, dH, dT, w);
    case GIST_STORE_F16:
      return run_copied<GIST_STORE_F16, GIST_STORE_F16>(st, D, p, H, nullptr, T, nullptr, labels, n_dev, loss, logp, lse, dH, dT, w);
    default:
      return run_copied<GIST_STORE_E4M3, GIST_STORE_E4M3>(st, D, p, H, h_scale, T, t_scale, labels, n_dev, loss, logp, lse, nullptr, nullptr, w);
  }
}

}  // namespace gist
