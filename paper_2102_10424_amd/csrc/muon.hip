// Orthogonalised updates: X = U / max(||U||_F, eps), then Newton-Schulz steps
//   A = X X^T,  B = b A + c A A,  X <- a X + B X
// on the fp16 matrix cores, and the weight update along the result.
//
// Operands.  |entries| <= singular values <= 8 (checked by the caller), so
// matrices are held times S = 2^12: fp16 then keeps 11 significant bits of
// entries from 2^-26 up, and all that is below 2^-37 is lost.  fp32 products hold
// every value in two parts, hi = fp16(v), lo = fp16(v - hi) (off by 2^-22 of the value
// and 2^-37) and take three products, hi hi' + hi lo' + lo hi'; lo lo' is at most
// 2^-22 of the product of the values.  With fp16 operands there is the one part, of 11 bits:
// X, A and B are rounded so in every step, which leaves the factor within 1.2e-3 of its norm.
// The parts are written by the kernel that produces a matrix, so the products
// load them as they are.  Matrices are padded with zeros to whole tiles, so
// that no product has edges: zero rows and columns stay zero.
//
// All three products are row times row (K contiguous in both operands): A and
// B are symmetric, and X is kept both as X (m x n) and as X^T (n x m), m <= n.
// Of A and B only the tiles on and below the diagonal are computed; the others
// are their mirror images.
//
// Layout: 128 bytes of a row hold 64 values, or 32 values' first and then second
// parts, so that a step of every product takes one 128-byte line of each row.

#include <algorithm>

#include "elem.cuh"

namespace gist {

namespace {

constexpr int kBlock = 256;
constexpr float kS = 4096.f, kInvS = 1.f / 4096.f;
constexpr int kNormBlocks = 512;

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef unsigned uintx2 __attribute__((ext_vector_type(2)));
typedef unsigned uintx4 __attribute__((ext_vector_type(4)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));

struct Update {
  float momentum, omu;   // omu = 1 - momentum
  float keep, eta;       // 1 - lr decay, lr scale
  int nesterov, fresh;
};

// ---- momentum and norm -----------------------------------------------------------

__device__ __forceinline__ float direction(const Update& u, float g, float m) {
  return u.nesterov ? fmaf(u.momentum, m, u.omu * g) : m;
}

// Sum over the workgroup, in a fixed order; every thread has it.
__device__ __forceinline__ double block_sum(double s, double* sh) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = s;
  __syncthreads();
  double r = 0.0;
  for (int w = 0; w < kBlock / 64; ++w) r += sh[w];
  return r;
}

// The new momentum, and per block the sum of squares of the direction, in
// double: part[group * kNormBlocks + block].  V floats a load: 4 where the
// groups' arrays are aligned.  Bound by memory: 71 us for three passes over two
// 4,096 x 4,096 matrices (5.7 TB/s), 159 with single floats and half the blocks.
template <bool UPDATE, int V>
__global__ __launch_bounds__(kBlock) void norm_kernel(int64_t count, const float* __restrict__ G,
                                                      float* __restrict__ M, Update u,
                                                      double* __restrict__ part) {
  __shared__ double sh[kBlock / 64];
  const int64_t off = blockIdx.y * count;
  constexpr int kUnroll = 4;
  const int64_t stride = static_cast<int64_t>(gridDim.x) * kBlock * V;
  double s = 0.0;
  for (int64_t e0 = (blockIdx.x * static_cast<int64_t>(kBlock) + threadIdx.x) * V; e0 < count; e0 += kUnroll * stride) {
    float v[kUnroll][V], m[kUnroll][V];
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
      const int64_t e = e0 + i * stride;
      if (e < count) {
        load_vec<GIST_STORE_F32, V>(G, off + e, v[i]);
        if (UPDATE && !u.fresh) load_vec<GIST_STORE_F32, V>(M, off + e, m[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
      const int64_t e = e0 + i * stride;
      if (e >= count) break;
#pragma unroll
      for (int q = 0; q < V; ++q) {
        if constexpr (UPDATE) {
          m[i][q] = fmaf(u.momentum, u.fresh ? 0.f : m[i][q], u.omu * v[i][q]);
          v[i][q] = direction(u, v[i][q], m[i][q]);
        }
        s += static_cast<double>(v[i][q]) * v[i][q];
      }
      if constexpr (UPDATE) store_vec<V>(M + off + e, m[i]);
    }
  }
  s = block_sum(s, sh);
  if (threadIdx.x == 0) part[blockIdx.y * kNormBlocks + blockIdx.x] = s;
}

template <int NP>
__device__ __forceinline__ void parts_of(float v, _Float16 (&p)[NP]) {
  p[0] = static_cast<_Float16>(v);
  if constexpr (NP == 2) p[1] = static_cast<_Float16>(v - static_cast<float>(p[0]));
}

// A matrix of ld values per row (a multiple of 64): part p of value j of row i
// is element at<NP>(i, j, p) of its group's block.
struct Mat {
  _Float16* p;
  int64_t ld, group;
};

template <int NP>
__device__ __forceinline__ int64_t at(const Mat& a, int64_t i, int64_t j, int p) {
  if constexpr (NP == 1) return i * a.ld + j;
  return 2 * i * a.ld + (j >> 5) * 64 + p * 32 + (j & 31);
}

// Eight consecutive values j..j+7 of row i (j a multiple of 8).
template <int NP>
__device__ __forceinline__ void put8(const Mat& a, int64_t g, int64_t i, int64_t j, const float (&v)[8]) {
  half8 h[NP];
#pragma unroll
  for (int q = 0; q < 8; ++q) {
    _Float16 s[NP];
    parts_of<NP>(v[q], s);
#pragma unroll
    for (int x = 0; x < NP; ++x) h[x][q] = s[x];
  }
#pragma unroll
  for (int x = 0; x < NP; ++x) *reinterpret_cast<half8*>(a.p + g * a.group + at<NP>(a, i, j, x)) = h[x];
}

template <int NP>
__device__ __forceinline__ void get8(const Mat& a, int64_t g, int64_t i, int64_t j, float (&v)[8]) {
  half8 h[NP];
#pragma unroll
  for (int x = 0; x < NP; ++x) h[x] = *reinterpret_cast<const half8*>(a.p + g * a.group + at<NP>(a, i, j, x));
#pragma unroll
  for (int q = 0; q < 8; ++q) {
    v[q] = static_cast<float>(h[0][q]);
    if constexpr (NP == 2) v[q] += static_cast<float>(h[1][q]);
  }
}

// Divisor of a group's matrix, from its partial sums: max(norm, eps), and a
// factor for both where the norm would not fit fp32.
struct Divisor {
  float pre, div;
};
__device__ __forceinline__ Divisor divisor_of(double squares, float eps) {
  double norm = sqrt(squares);
  Divisor d{1.f, 0.f};
  if (norm > 1e30) {
    d.pre = 0x1p-64f;
    norm *= 0x1p-64;
  }
  d.div = norm < static_cast<double>(eps) ? eps : static_cast<float>(norm);   // NaN stays
  return d;
}
__device__ __forceinline__ Divisor divisor(const double* __restrict__ part, int64_t g, int nparts, float eps,
                                           double* sh) {
  double s = 0.0;
  for (int i = threadIdx.x; i < nparts; i += kBlock) s += part[g * kNormBlocks + i];
  return divisor_of(block_sum(s, sh), eps);
}

// U / norm, split, as it stands (D) and transposed (T); 64 x 64 tiles over the
// padded sides, 16 values of a row per thread.  Bound by memory: 130 us for two 4,096 x
// 4,096 matrices with momentum (537 MB, 4.1 TB/s).
template <bool UPDATE, int NP, bool VEC>
__global__ __launch_bounds__(kBlock) void split_kernel(int64_t rows, int64_t cols, int nparts,
                                                       const float* __restrict__ G,
                                                       const float* __restrict__ M, Update u,
                                                       const double* __restrict__ part, float eps,
                                                       Mat D, Mat T) {
  __shared__ double red[kBlock / 64];
  __shared__ __attribute__((aligned(8))) float tile[64][66];   // 66: column reads spread over the banks
  const int t = threadIdx.x;
  const int64_t g = blockIdx.z, off = g * rows * cols;
  const int64_t r0 = blockIdx.y * 64, c0 = blockIdx.x * 64;
  const int r = t >> 2, c = (t & 3) * 16;
  float v[16];
#pragma unroll
  for (int q = 0; q < 16; ++q) v[q] = 0.f;
  if (r0 + r < rows) {
    const int64_t e = off + (r0 + r) * cols + c0 + c;
#pragma unroll
    for (int q = 0; q < 16; q += 4) {
      float x[4] = {}, m[4] = {};
      if constexpr (VEC) {   // cols is a multiple of 4
        if (c0 + c + q < cols) {
          load_vec<GIST_STORE_F32, 4>(G, e + q, x);
          if (UPDATE) load_vec<GIST_STORE_F32, 4>(M, e + q, m);
        }
      } else {
#pragma unroll
        for (int y = 0; y < 4; ++y)
          if (c0 + c + q + y < cols) {
            x[y] = G[e + q + y];
            if (UPDATE) m[y] = M[e + q + y];
          }
      }
#pragma unroll
      for (int y = 0; y < 4; ++y) v[q + y] = UPDATE ? direction(u, x[y], m[y]) : x[y];
    }
  }
  const Divisor d = divisor(part, g, nparts, eps, red);
#pragma unroll
  for (int h = 0; h < 16; h += 8) {
    float x[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) x[q] = kS * (v[h + q] * d.pre / d.div);
    put8<NP>(D, g, r0 + r, c0 + c + h, x);
#pragma unroll
    for (int q = 0; q < 8; q += 2) *reinterpret_cast<floatx2*>(&tile[r][c + h + q]) = floatx2{x[q], x[q + 1]};
  }
  __syncthreads();
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int j = (t >> 3) + 32 * h, p = (t & 7) * 8;   // column j, rows p..p+7
    float x[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) x[q] = tile[p + q][j];
    put8<NP>(T, g, c0 + j, r0 + p, x);
  }
}

// ---- products ------------------------------------------------------------------------

enum { kGram = 0, kPoly = 1, kStep = 2, kLast = 3 };

struct Epi {
  Mat out, outT;          // kGram, kPoly: out; kStep: both
  Mat add;                // kPoly: A; kStep, kLast: X
  float alpha, beta;      // out = alpha * add + beta * product
  float* W;               // kLast: weights, or
  void* O;                // the factor itself
  int64_t m, n;           // kLast: sizes without padding
  int64_t si, sj, group;  // kLast: element (i, j) at i * si + j * sj
  float keep, eta;
  int o_half;
  int vec;                // kLast: eight consecutive elements are 16-byte aligned
};

// Workgroup barrier that orders LDS only.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Wait until at most N of this wave's loads are out (the counter takes 6 bits).
template <int N>
__device__ __forceinline__ void wait_loads() {
  static_assert(N >= 0 && N < 64, "vmcnt");
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// 16 bytes per lane from memory straight to LDS: base + off (per lane) to
// dst + 16 lane.  No vector register is written; the caller waits for vmcnt.
// (m0, which holds dst, is a register the compiler reserves, of which it warns.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_to_lds(unsigned dst, unsigned off, const char* base) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :
               : "s"(dst), "v"(off), "s"(base)
               : "memory", "m0");
}
#pragma clang diagnostic pop

// Work of one product: tiles of all groups.  The first `whole` are one
// workgroup's each; the others (`ragged` of them) are cut in K into `slices`
// of `len` steps, slice-major, joined by a second kernel.
struct Sched {
  int tiles_m, tiles_n, tiles;   // of one matrix
  int64_t whole, ragged;
  int slices, len, steps;
};

// Tile t of the lower triangle, row by row.
__device__ __forceinline__ void triangle(int t, int& ti, int& tj) {
  ti = static_cast<int>((sqrtf(8.f * t + 1.f) - 1.f) * 0.5f);
  while (ti * (ti + 1) / 2 > t) --ti;
  while ((ti + 1) * (ti + 2) / 2 <= t) ++ti;
  tj = t - ti * (ti + 1) / 2;
}

template <int MODE>
__device__ __forceinline__ void tile_of(const Sched& S, int64_t id, int64_t& g, int& ti, int& tj) {
  g = static_cast<unsigned>(id) / static_cast<unsigned>(S.tiles);
  const int x = static_cast<int>(id - g * S.tiles);
  if constexpr (MODE == kGram || MODE == kPoly) {
    triangle(x, ti, tj);
  } else {
    ti = x % S.tiles_m;
    tj = x / S.tiles_m;
  }
}

// The weights' step, or the factor, for eight consecutive elements from e on,
// the first `left` of them in the matrix.
__device__ __forceinline__ void last8(const Epi& E, int64_t e, int left, const float (&v)[8]) {
  if (left <= 0) return;
  if (E.vec && left >= 8) {
    if (!E.W && E.o_half) {
      half8 h;
#pragma unroll
      for (int q = 0; q < 8; ++q) h[q] = static_cast<_Float16>(v[q] * kInvS);
      *reinterpret_cast<half8*>(static_cast<_Float16*>(E.O) + e) = h;
      return;
    }
#pragma unroll
    for (int h = 0; h < 8; h += 4) {
      floatx4* p = reinterpret_cast<floatx4*>((E.W ? E.W : static_cast<float*>(E.O)) + e + h);
      floatx4 w;
      if (E.W) w = *p;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float o = v[h + q] * kInvS;
        w[q] = E.W ? fmaf(-E.eta, o, E.keep * w[q]) : o;
      }
      *p = w;
    }
    return;
  }
#pragma unroll
  for (int q = 0; q < 8; ++q) {
    if (q >= left) break;
    const float o = v[q] * kInvS;
    if (E.W) E.W[e + q] = fmaf(-E.eta, o, E.keep * E.W[e + q]);
    else if (E.o_half) static_cast<_Float16*>(E.O)[e + q] = static_cast<_Float16>(o);
    else static_cast<float*>(E.O)[e + q] = o;
  }
}

// One 32 x 32 block at (row, col) of group g's result.  Accumulator register r
// of lane l: row 8 (r / 4) + 4 (l / 32) + r mod 4, column l mod 32.  The block
// goes through the wave's own LDS (32 rows of 34 floats), so that memory sees
// 16 bytes per lane both for the rows and for the columns of the result:
// element by element, the loads and stores of a 256 x 256 tile kept the load
// path busy for 40 us.
constexpr int kScratch = 32 * 34;
template <int NP, int MODE>
__device__ __forceinline__ void finish_block(const floatx16& acc, const Epi& E, int64_t g, int row, int col,
                                             int lane, float* sc) {
  if ((MODE == kGram || MODE == kPoly) && row < col) return;   // the mirror image of another block
  wave_sync();   // the last block's values are read
#pragma unroll
  for (int r = 0; r < 16; ++r)   // the product times S
    sc[(8 * (r >> 2) + 4 * (lane >> 5) + (r & 3)) * 34 + (lane & 31)] = acc[r] * kInvS;
  wave_sync();
  const bool rows = MODE != kLast || E.sj == 1;
  const bool cols = MODE == kStep || (MODE == kLast ? E.sj != 1 : row != col);
  const int p = 8 * (lane & 3);
#pragma unroll
  for (int it = 0; it < 2; ++it) {
    const int i = it * 16 + (lane >> 2);
    float v[8];
#pragma unroll
    for (int q = 0; q < 8; q += 2) {
      const floatx2 x = *reinterpret_cast<const floatx2*>(sc + i * 34 + p + q);
      v[q] = x[0];
      v[q + 1] = x[1];
    }
    if constexpr (MODE != kGram) {
      float o[8];
      get8<NP>(E.add, g, row + i, col + p, o);
#pragma unroll
      for (int q = 0; q < 8; ++q) v[q] = fmaf(E.alpha, o[q], E.beta * v[q]);
      if (cols) {
#pragma unroll
        for (int q = 0; q < 8; q += 2) *reinterpret_cast<floatx2*>(sc + i * 34 + p + q) = floatx2{v[q], v[q + 1]};
      }
    }
    if constexpr (MODE == kLast) {
      if (rows && row + i < E.m)
        last8(E, g * E.group + (row + i) * E.si + col + p, static_cast<int>(E.n) - col - p, v);
    } else {
      put8<NP>(E.out, g, row + i, col + p, v);
    }
  }
  if (!cols) return;
  wave_sync();
#pragma unroll
  for (int it = 0; it < 2; ++it) {
    const int j = it * 16 + (lane >> 2);
    float v[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] = sc[(p + q) * 34 + j];
    if constexpr (MODE == kLast) {
      if (col + j < E.n)
        last8(E, g * E.group + (col + j) * E.sj + row + p, static_cast<int>(E.m) - row - p, v);
    } else {
      put8<NP>(MODE == kStep ? E.outT : E.out, g, col + j, row + p, v);
    }
  }
}

// P Q^T (rows of both K contiguous), tiles of 32 WM NWM x 32 WN NWN by NWM x NWN
// waves.  Every step takes 128 bytes of each of the tile's rows: lines go
// from memory to one of two LDS buffers while the matrix cores work on the
// other; one barrier per step.  A row's eight 16-byte pieces lie in LDS in the
// order piece ^ (row / 2 mod 8), which spreads a fragment read (one piece of 32
// rows) over the 64 banks; the lanes of the load pick their piece accordingly.
// (By row mod 8, right for 32 banks, half of all LDS cycles were conflicts.)
// NS buffers; small tiles, whose steps are short, need more of them to cover
// memory's latency.
// What bounds it: power for large matrices (the clock falls to 1.8 GHz with the matrix
// cores busy 57% of the cycles; half of the LDS cycles less, or 4 waves of 128 x 128 with
// a third less LDS traffic, made no difference), 700-740 us for two products of 4,096
// cubed in two parts each (1,110-1,180 fp16 TFLOP/s, a library's fp16 product 1,240) and
// 131 us for one of one part (1,050); latency for small ones, about 5 us a launch.
template <int NP, int MODE, int WM, int WN, int NWM, int NWN, int NS>
__global__ __launch_bounds__(64 * NWM * NWN, 2) void product_kernel(Sched S, Mat P, Mat Q, Epi E,
                                                                    float* __restrict__ part) {
  constexpr int BM = 32 * WM * NWM, BN = 32 * WN * NWN;
  constexpr int ROWS = BM + BN, LOADS = ROWS / 8 / (NWM * NWN);   // 8 rows a wave's load
  constexpr int QN = 4 / NP;                                       // MFMA depths (16 values) per step
  __shared__ __attribute__((aligned(1024))) char lds[NS][ROWS * 128];
  const int t = threadIdx.x, lane = t & 63;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int li = lane & 31, lh = lane >> 5;
  const int wm = wave / NWN, wn = wave % NWN;
  int64_t id, u = -1, g;
  int ti, tj, k0 = 0, steps = S.steps;
  if (blockIdx.x < S.whole) {
    id = xcd_remap(blockIdx.x, S.whole);
  } else {
    u = xcd_remap(blockIdx.x - S.whole, gridDim.x - S.whole);
    const int slice = static_cast<int>(static_cast<unsigned>(u) / static_cast<unsigned>(S.ragged));
    id = S.whole + (u - slice * S.ragged);
    k0 = slice * S.len;
    steps = min(S.len, S.steps - k0);
  }
  tile_of<MODE>(S, id, g, ti, tj);
  const int64_t ldp = P.ld * (2 * NP), ldq = Q.ld * (2 * NP);   // bytes
  const char* const pb = reinterpret_cast<const char*>(P.p + g * P.group) + ti * BM * ldp + k0 * 128;
  const char* const qb = reinterpret_cast<const char*>(Q.p + g * Q.group) + tj * BN * ldq + k0 * 128;
  const unsigned lds0 = static_cast<unsigned>(reinterpret_cast<uintptr_t>(
      (__attribute__((address_space(3))) char*)&lds[0][0]));
  static_assert(LOADS % 2 == 0, "the piece order below goes by the parity of a load");
  unsigned offp[2], offq[2];   // of even and odd loads
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const unsigned piece = ((lane & 7) ^ ((lane >> 4) + 4 * h)) * 16;
    offp[h] = static_cast<unsigned>((lane >> 3) * ldp) + piece;
    offq[h] = static_cast<unsigned>((lane >> 3) * ldq) + piece;
  }
  auto load = [&](int buf, int j, int i) {   // the wave's load i of step j
    const int r = (wave * LOADS + i) * 8;    // first of its eight rows (P's, then Q's)
    const bool p = r < BM;
    const char* base = p ? pb + r * ldp : qb + (r - BM) * ldq;
    load_to_lds(lds0 + buf * (ROWS * 128) + r * 128, p ? offp[i & 1] : offq[i & 1], base + j * 128);
  };
  floatx16 acc[WM][WN] = {};
#pragma unroll
  for (int j = 0; j < NS; ++j) {
    const int js = min(j, steps - 1);   // always NS steps' loads, so that the counts below hold
#pragma unroll
    for (int i = 0; i < LOADS; ++i) load(j, js, i);
  }
  const char* const fa = &lds[0][0] + (wm * WM * 32 + li) * 128;
  const char* const fb = &lds[0][0] + (BM + wn * WN * 32 + li) * 128;
  int fo[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) fo[q] = ((2 * q + lh) ^ (li >> 1 & 7)) * 16;
  half8 a[2][WM][NP], b[2][WN][NP];   // fragments of this depth and of the next
  auto read = [&](int to, int buf, int q) {
    const int bo = buf * (ROWS * 128);
#pragma unroll
    for (int s = 0; s < NP; ++s) {
#pragma unroll
      for (int x = 0; x < WM; ++x)
        a[to][x][s] = *reinterpret_cast<const half8*>(fa + bo + x * 4096 + fo[2 * s + q]);
#pragma unroll
      for (int x = 0; x < WN; ++x)
        b[to][x][s] = *reinterpret_cast<const half8*>(fb + bo + x * 4096 + fo[2 * s + q]);
    }
  };
  wait_loads<LOADS * (NS - 1)>();
  lds_barrier();
  read(0, 0, 0);
  int buf = 0, next = 1 % NS;
  for (int j = 0; j < steps; ++j) {
#pragma unroll
    for (int q = 0; q < QN; ++q) {
      const int f = q & 1;
      if (q + 1 < QN) {
        read(f ^ 1, buf, q + 1);
      } else {
        // The last depth of step j: its buffer has been read by this wave, and
        // behind the barrier by all, so it takes step j + NS; step j + 1 has
        // arrived when at most NS - 2 steps' loads are out.  Its first
        // fragments are read while the matrix cores still work on step j.
        wait_loads<LOADS * (NS - 2)>();
        lds_barrier();
        const int js = min(j + NS, steps - 1);   // past the end: the last step again, never used
#pragma unroll
        for (int i = 0; i < LOADS; ++i) load(buf, js, i);
        read(f ^ 1, next, 0);
      }
      if constexpr (NP == 2) {
#pragma unroll
        for (int x = 0; x < WM; ++x)
#pragma unroll
          for (int y = 0; y < WN; ++y)
            acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[f][x][0], b[f][y][1], acc[x][y], 0, 0, 0);
#pragma unroll
        for (int x = 0; x < WM; ++x)
#pragma unroll
          for (int y = 0; y < WN; ++y)
            acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[f][x][1], b[f][y][0], acc[x][y], 0, 0, 0);
      }
#pragma unroll
      for (int x = 0; x < WM; ++x)
#pragma unroll
        for (int y = 0; y < WN; ++y)
          acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[f][x][0], b[f][y][0], acc[x][y], 0, 0, 0);
#pragma unroll
      for (int m = 0; m < WM * WN * (NP == 2 ? 3 : 1); ++m) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);   // an MFMA
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);   // an LDS read
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    buf = next;
    next = next + 1 == NS ? 0 : next + 1;
  }
  wait_loads<0>();   // nothing may still be on its way to LDS when the workgroup ends
  if (u >= 0) {   // a slice: its sums, 32 x 32 blocks in accumulator order
    floatx4* d = reinterpret_cast<floatx4*>(part + u * static_cast<int64_t>(BM * BN)) + lane;
#pragma unroll
    for (int x = 0; x < WM; ++x)
#pragma unroll
      for (int y = 0; y < WN; ++y)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
          const int blk = (wm * WM + x) * (BN / 32) + wn * WN + y;
          d[(blk * 4 + r4) * 64] = floatx4{acc[x][y][4 * r4], acc[x][y][4 * r4 + 1], acc[x][y][4 * r4 + 2],
                                           acc[x][y][4 * r4 + 3]};
        }
    return;
  }
  lds_barrier();   // every wave is done with its fragments: their LDS serves finish_block
  float* const sc = reinterpret_cast<float*>(&lds[0][0]) + wave * kScratch;
  static_assert(sizeof(lds) >= NWM * NWN * kScratch * 4, "scratch of all waves");
#pragma unroll
  for (int x = 0; x < WM; ++x)
#pragma unroll
    for (int y = 0; y < WN; ++y)
      finish_block<NP, MODE>(acc[x][y], E, g, ti * BM + (wm * WM + x) * 32, tj * BN + (wn * WN + y) * 32,
                             lane, sc);
}

// Tiles that were cut in K: a wave per 32 x 32 block adds the slices in order
// (16 tiles of 256 x 256 in eight slices 9 us; uncut, they were a round of 290).
template <int NP, int MODE, int TILE>
__global__ __launch_bounds__(kBlock) void join_kernel(Sched S, const float* __restrict__ part, Epi E) {
  __shared__ __attribute__((aligned(16))) float scratch[kBlock / 64][kScratch];
  constexpr int NB = TILE / 32, BLOCKS = NB * NB;
  const int lane = threadIdx.x & 63;
  const int64_t w = (static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x) >> 6;
  const int blk = static_cast<int>(w % BLOCKS);
  const int64_t rt = w / BLOCKS;
  if (rt >= S.ragged) return;
  int64_t g;
  int ti, tj;
  tile_of<MODE>(S, S.whole + rt, g, ti, tj);
  floatx16 acc = {};
  for (int s = 0; s < S.slices; ++s) {
    const floatx4* d = reinterpret_cast<const floatx4*>(part + (s * S.ragged + rt) * (TILE * TILE)) + blk * 256 + lane;
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      const floatx4 v = d[r4 * 64];
#pragma unroll
      for (int q = 0; q < 4; ++q) acc[4 * r4 + q] += v[q];
    }
  }
  finish_block<NP, MODE>(acc, E, g, ti * TILE + (blk / NB) * 32, tj * TILE + (blk % NB) * 32, lane,
                         scratch[threadIdx.x >> 6]);
}

// ---- matrices with a side of up to 128 -------------------------------------------------
//
// A workgroup keeps a slab of 128 columns of X (both ways round) in LDS, computes
// A and B itself and steps its slab; slabs meet only in A, whose parts (one per
// slab) go through memory from one launch to the next.  So a step is one launch
// instead of three, and one slab (n <= 128) takes all steps in one.
// B = b A + c A A is symmetric: a block B[k][r] as an MFMA result, lane = column r,
// four k in a lane's registers, is B[r][k] in the layout of an MFMA operand but for
// which half of the wave holds which four of eight k.

constexpr int kSlab = 128, kSmallThreads = 512, kSmallWaves = 8;

struct SmallArgs {
  int64_t rows, cols;
  int m, n, slabs, flip;
  const float* G;
  float *M, *W;
  void* O;
  Update u;
  const double* norm;      // sums of squares (slabs > 1)
  int nparts;
  float eps, ca, cb, cc;
  int first, k0, k1, steps;
  const float* pin;        // A's parts of the last launch
  float* pout;
  char* T;                 // the slabs between launches, as they lie in LDS
};

// Byte of value k, part p in a row, and its place: pieces of 16 bytes in an order
// that spreads a column of rows over the banks.
template <int NP, int RB>
__device__ __forceinline__ int small_at(int row, int k, int p) {
  const int byte = NP == 1 ? 2 * k : (k >> 5) * 128 + p * 64 + (k & 31) * 2;
  const int swz = RB >= 256 ? row & 15 : row >> 1 & 7;
  return row * RB + (((byte >> 4) ^ swz) << 4) + (byte & 15);
}
// The same for an MFMA fragment (row li of a block of 32, k = 16 d + 8 lh): a lane's
// base, into which depth and part go by exclusive or; blocks are 32 RB apart.
template <int RB>
__device__ __forceinline__ int small_base(int li, int lh) {
  return li * RB + (((RB >= 256 ? li & 15 : li >> 1 & 7) ^ lh) << 4);
}
// A copy the compiler cannot see through: addresses are then formed where they are
// used, rather than kept, by the dozen, in registers across the loop.
__device__ __forceinline__ int fresh(int x) {
  asm volatile("" : "+v"(x));
  return x;
}
template <int NP>
__device__ __forceinline__ void small_frag(const char* r, int base, int d, half8 (&f)[NP]) {
#pragma unroll
  for (int p = 0; p < NP; ++p)
    f[p] = *reinterpret_cast<const half8*>(r + (base ^ (NP == 1 ? 32 * d : (d >> 1) * 128 + p * 64 + (d & 1) * 32)));
}
// Four consecutive values k .. k + 3 of row li, k = K0 + 8 r4 + 4 lh with K0 a multiple
// of 32: a lane's base and, by exclusive or, K0, r4 and the part.
template <int RB>
__device__ __forceinline__ int quad_base(int li, int lh) {
  return li * RB + ((RB >= 256 ? li & 15 : li >> 1 & 7) << 4) + 8 * lh;
}
template <int NP>
__device__ __forceinline__ int quad_at(int k0, int r4, int p) {
  return (NP == 1 ? 2 * k0 : 4 * k0 + 64 * p) + 16 * r4;
}
// One value of row R0 + 8 r4 + 4 lh + q (R0 a multiple of 32) at k = K0 + li.
template <int RB>
__device__ __forceinline__ int cross_base(int li, int lh) {
  return 4 * lh * RB + (((li >> 3) ^ (RB >= 256 ? 4 * lh : 2 * lh)) << 4) + (li & 7) * 2;
}
template <int NP, int RB>
__device__ __forceinline__ int cross_at(int k0, int r4, int q, int p) {
  return (NP == 1 ? 2 * k0 : 4 * k0 + 64 * p) ^ ((RB >= 256 ? 8 * (r4 & 1) + q : 4 * (r4 & 1) + (q >> 1)) << 4);
}
template <int NP>
__device__ __forceinline__ floatx4 get_quad(const char* r, int base, int k0, int r4) {
  floatx4 v = __builtin_convertvector(*reinterpret_cast<const half4*>(r + (base ^ quad_at<NP>(k0, r4, 0))), floatx4);
  if constexpr (NP == 2)
    v += __builtin_convertvector(*reinterpret_cast<const half4*>(r + (base ^ quad_at<NP>(k0, r4, 1))), floatx4);
  return v;
}
template <int NP>
__device__ __forceinline__ void split4(floatx4 v, half4 (&h)[NP]) {
  h[0] = __builtin_convertvector(v, half4);
  if constexpr (NP == 2) h[1] = __builtin_convertvector(v - __builtin_convertvector(h[0], floatx4), half4);
}
template <int NP>
__device__ __forceinline__ void put_quad(char* r, int base, int k0, int r4, const half4 (&h)[NP]) {
#pragma unroll
  for (int p = 0; p < NP; ++p) *reinterpret_cast<half4*>(r + (base ^ quad_at<NP>(k0, r4, p))) = h[p];
}
// The four as values of four rows (r: the first row's block).
template <int NP, int RB>
__device__ __forceinline__ void put_cross(char* r, int base, int k0, int r4, const half4 (&h)[NP]) {
#pragma unroll
  for (int p = 0; p < NP; ++p)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *reinterpret_cast<_Float16*>(r + (8 * r4 + q) * RB + (base ^ cross_at<NP, RB>(k0, r4, q, p))) = h[p][q];
}
template <int NP, int RB>
__device__ __forceinline__ void small_put1(char* r, int row, int k, float v) {
  _Float16 s[NP];
  parts_of<NP>(v, s);
#pragma unroll
  for (int p = 0; p < NP; ++p) *reinterpret_cast<_Float16*>(r + small_at<NP, RB>(row, k, p)) = s[p];
}
template <int NP>
__device__ __forceinline__ void mma(floatx16& acc, const half8 (&a)[NP], const half8 (&b)[NP]) {
  if constexpr (NP == 2) {
    acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[0], b[1], acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[1], b[0], acc, 0, 0, 0);
  }
  acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[0], b[0], acc, 0, 0, 0);
}
// Block b of the lower triangle of blocks, row by row.
__device__ __forceinline__ void lower_block(int b, int& rb, int& cb) {
  rb = b < 1 ? 0 : b < 3 ? 1 : b < 6 ? 2 : 3;
  cb = b - rb * (rb + 1) / 2;
}

template <int NP, int MP, bool UPDATE>
__global__ __launch_bounds__(kSmallThreads, 2) void small_kernel(SmallArgs a) {
  constexpr int RT = MP * NP * 2, RX = kSlab * NP * 2;      // bytes of a row of A and X^T, of X
  constexpr int NRB = MP / 32, LOW = NRB * (NRB + 1) / 2;   // 32-row blocks, blocks of the lower triangle
  constexpr int KD = MP / 16, NB = NRB / 2;                 // depths of K = MP, column blocks per wave
  constexpr int OWN = (LOW + kSmallWaves - 1) / kSmallWaves;
  constexpr int KPG = NRB * NRB > kSmallWaves ? NRB * NRB / kSmallWaves : 1;   // blocks of B per wave
  __shared__ __attribute__((aligned(16))) char ra[MP * RX];   // A (RT <= RX), then the new X
  __shared__ __attribute__((aligned(16))) char rt[kSlab * RT];
  __shared__ double red[kSmallWaves];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, li = lane & 31, lh = lane >> 5;
  const int slab = blockIdx.x;
  const int64_t g = blockIdx.y, off = g * a.rows * a.cols;
  const int rb = wave % NRB, cg = wave / NRB;
  auto elem = [&](int i, int j) { return off + (a.flip ? (slab * kSlab + j) * a.cols + i : i * a.cols + slab * kSlab + j); };
  char* const tg = a.T + (g * a.slabs + slab) * (kSlab * RT);
  float* const pout = a.pout + (g * a.slabs + slab) * (LOW * 1024);
  floatx16 low[OWN];   // this wave's blocks of A

  // A's blocks, to LDS: both triangles.
  auto put_a = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < OWN; ++x) {
      const int b = wave + x * kSmallWaves;
      if (b >= LOW) continue;
      int br, bc;
      lower_block(b, br, bc);
      const int qb = fresh(quad_base<RT>(li, lh)), xb = fresh(cross_base<RT>(li, lh));
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        half4 h[NP];
        split4<NP>(floatx4{low[x][4 * r4], low[x][4 * r4 + 1], low[x][4 * r4 + 2], low[x][4 * r4 + 3]} * kInvS, h);
        put_quad<NP>(ra + bc * 32 * RT, qb, br * 32, r4, h);
        if (br != bc) put_cross<NP, RT>(ra + br * 32 * RT, xb, bc * 32, r4, h);
      }
    }
  };
  // A's blocks from X, to the last part of K this slab has.
  auto gram = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < OWN; ++x) {
      const int b = wave + x * kSmallWaves;
      low[x] = floatx16{};
      if (b >= LOW) continue;
      int br, bc;
      lower_block(b, br, bc);
      const int fb = fresh(small_base<RX>(li, lh));
#pragma unroll
      for (int d = 0; d < kSlab / 16; ++d) {
        half8 p[NP], q[NP];
        small_frag<NP>(ra + br * 32 * RX, fb, d, p);
        small_frag<NP>(ra + bc * 32 * RX, fb, d, q);
        mma<NP>(low[x], p, q);
        if (d & 1) __builtin_amdgcn_sched_barrier(0);   // else all reads come first, into too many registers
      }
    }
    if (a.slabs == 1) {
      __syncthreads();   // X is read: A takes its place
      put_a();
    } else {
#pragma unroll
      for (int x = 0; x < OWN; ++x) {
        const int b = wave + x * kSmallWaves;
        if (b >= LOW) continue;
        floatx4* d = reinterpret_cast<floatx4*>(pout + b * 1024) + lane;
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4)
          d[r4 * 64] = floatx4{low[x][4 * r4], low[x][4 * r4 + 1], low[x][4 * r4 + 2], low[x][4 * r4 + 3]};
      }
    }
  };
  auto save_slab = [&]() __attribute__((always_inline)) {
    for (int x = t * 16; x < kSlab * RT; x += kSmallThreads * 16)
      *reinterpret_cast<uint4*>(tg + x) = *reinterpret_cast<const uint4*>(rt + x);
  };

  if (a.first) {
    constexpr int PER = MP * kSlab / kSmallThreads;
    float v[PER], mo[UPDATE ? PER : 1];
    auto place = [&](int x, int& i, int& j) __attribute__((always_inline)) {   // in the matrix?
      const int e = x * kSmallThreads + t;
      i = a.flip ? e & (MP - 1) : e / kSlab;
      j = a.flip ? e / MP : e & (kSlab - 1);
      return i < a.m && slab * kSlab + j < a.n;
    };
    // every load is made, at the group's first element outside the matrix: none waits for
    // another behind a branch
#pragma unroll
    for (int x = 0; x < PER; ++x) {
      int i, j;
      const int64_t at = place(x, i, j) ? elem(i, j) : off;
      v[x] = a.G[at];
      if constexpr (UPDATE) mo[x] = a.u.fresh && a.slabs == 1 ? 0.f : a.M[at];
    }
    double s = 0.0;
#pragma unroll
    for (int x = 0; x < PER; ++x) {
      int i, j;
      const bool in = place(x, i, j);
      if constexpr (UPDATE) {
        if (a.slabs == 1) {   // else norm_kernel has stepped it
          mo[x] = fmaf(a.u.momentum, mo[x], a.u.omu * v[x]);
          if (in) a.M[elem(i, j)] = mo[x];
        }
        v[x] = direction(a.u, v[x], mo[x]);
      }
      if (!in) v[x] = 0.f;
      s += static_cast<double>(v[x]) * v[x];
    }
    if (a.slabs > 1) {
      s = 0.0;
      for (int x = t; x < a.nparts; x += kSmallThreads) s += a.norm[g * kNormBlocks + x];
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    if (lane == 0) red[wave] = s;
    __syncthreads();
    s = 0.0;
    for (int w = 0; w < kSmallWaves; ++w) s += red[w];
    const Divisor dv = divisor_of(s, a.eps);
#pragma unroll
    for (int x = 0; x < PER; ++x) {
      int i, j;
      place(x, i, j);
      const float y = kS * (v[x] * dv.pre / dv.div);
      small_put1<NP, RT>(rt, j, i, y);
      small_put1<NP, RX>(ra, i, j, y);
    }
    __syncthreads();
    gram();
    if (a.slabs > 1) save_slab();
  } else {
    for (int x = t * 16; x < kSlab * RT; x += kSmallThreads * 16)
      *reinterpret_cast<uint4*>(rt + x) = *reinterpret_cast<const uint4*>(tg + x);
    // A: the slabs' parts, in order
#pragma unroll
    for (int x = 0; x < OWN; ++x) {
      const int b = wave + x * kSmallWaves;
      low[x] = floatx16{};
      if (b >= LOW) continue;
      const floatx4* d = reinterpret_cast<const floatx4*>(a.pin + g * a.slabs * (LOW * 1024) + b * 1024) + lane;
#pragma unroll 4
      for (int y = 0; y < a.slabs; ++y) {
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
          const floatx4 w = d[y * (LOW * 256) + r4 * 64];
#pragma unroll
          for (int q = 0; q < 4; ++q) low[x][4 * r4 + q] += w[q];
        }
      }
    }
    put_a();
  }
  for (int k = a.k0; k < a.k1; ++k) {
    __syncthreads();
    // B: a wave computes KPG of its rows' blocks and the waves of the same rows trade
    // them through LDS, in A's place
    half4 mine[KPG][4][NP];
    if (cg < NRB / KPG) {
#pragma unroll
      for (int x = 0; x < KPG; ++x) {
        const int kb = cg * KPG + x;
        floatx16 acc = {};
        const int fb = fresh(small_base<RT>(li, lh));
#pragma unroll
        for (int d = 0; d < KD; ++d) {
          half8 p[NP], q[NP];
          small_frag<NP>(ra + kb * 32 * RT, fb, d, p);
          small_frag<NP>(ra + rb * 32 * RT, fb, d, q);
          mma<NP>(acc, p, q);
          if (d & 1) __builtin_amdgcn_sched_barrier(0);
        }
        const int qb = fresh(quad_base<RT>(li, lh));
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
          const floatx4 v = get_quad<NP>(ra + rb * 32 * RT, qb, kb * 32, r4);
          const floatx4 c = floatx4{acc[4 * r4], acc[4 * r4 + 1], acc[4 * r4 + 2], acc[4 * r4 + 3]} * (a.cc * kInvS);
          split4<NP>(a.cb * v + c, mine[x][r4]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    __syncthreads();   // A is read
    // depth d, part p of rows rb: 1 KB at ((rb KD + d) NP + p), a lane's 16 bytes (eight k) in
    // two halves: k 0..3 from the lower half of the wave, 4..7 from the upper
    if (cg < NRB / KPG) {
#pragma unroll
      for (int x = 0; x < KPG; ++x)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4)
#pragma unroll
          for (int p = 0; p < NP; ++p) {
            const int d = 2 * (cg * KPG + x) + (r4 >> 1);
            *reinterpret_cast<half4*>(ra + (((rb * KD + d) * NP + p) * 64 + (r4 & 1) * 32 + li) * 16 + lh * 8) = mine[x][r4][p];
          }
    }
    __syncthreads();
    half8 B[KD][NP];   // rows rb of B
#pragma unroll
    for (int d = 0; d < KD; ++d)
#pragma unroll
      for (int p = 0; p < NP; ++p)
        B[d][p] = *reinterpret_cast<const half8*>(ra + (((rb * KD + d) * NP + p) * 64 + lane) * 16);
    floatx4 v[NB][4];
#pragma unroll
    for (int y = 0; y < NB; ++y) {
      const char* const tr = rt + (cg * NB + y) * 32 * RT;
      const int fb = fresh(small_base<RT>(li, lh)), qb = fresh(quad_base<RT>(li, lh));
      floatx16 acc = {};
#pragma unroll
      for (int d = 0; d < KD; ++d) {
        half8 q[NP];
        small_frag<NP>(tr, fb, d, q);
        mma<NP>(acc, B[d], q);
        if (d & 1) __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4)
        v[y][r4] = a.ca * get_quad<NP>(tr, qb, rb * 32, r4) +
                   floatx4{acc[4 * r4], acc[4 * r4 + 1], acc[4 * r4 + 2], acc[4 * r4 + 3]} * kInvS;
      __builtin_amdgcn_sched_barrier(0);
    }
    if (k + 1 == a.steps) {
#pragma unroll
      for (int y = 0; y < NB; ++y) {
        const int j = (cg * NB + y) * 32 + li;
        const bool jn = slab * kSlab + j < a.n;
        float w[4][4];
        if constexpr (UPDATE) {
#pragma unroll
          for (int r4 = 0; r4 < 4; ++r4)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const int i = rb * 32 + 8 * r4 + 4 * lh + q;
              w[r4][q] = a.W[jn && i < a.m ? elem(i, j) : off];
            }
        }
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int i = rb * 32 + 8 * r4 + 4 * lh + q;
            const float o = v[y][r4][q] * kInvS;
            if (jn && i < a.m) {
              const int64_t e = elem(i, j);
              if constexpr (UPDATE) a.W[e] = fmaf(-a.u.eta, o, a.u.keep * w[r4][q]);
              else if constexpr (NP == 1) static_cast<_Float16*>(a.O)[e] = static_cast<_Float16>(o);
              else static_cast<float*>(a.O)[e] = o;
            }
          }
      }
      return;
    }
    __syncthreads();   // A and X^T are read
#pragma unroll
    for (int y = 0; y < NB; ++y) {
      const int qb = fresh(quad_base<RT>(li, lh)), xb = fresh(cross_base<RX>(li, lh));
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        half4 h[NP];
        split4<NP>(v[y][r4], h);
        put_quad<NP>(rt + (cg * NB + y) * 32 * RT, qb, rb * 32, r4, h);
        put_cross<NP, RX>(ra + rb * 32 * RX, xb, (cg * NB + y) * 32, r4, h);
      }
    }
    __syncthreads();
    gram();
    if (a.slabs > 1) save_slab();
  }
}

size_t up256(size_t x) { return (x + 255) & ~size_t(255); }

// The tiles: side, workgroups the card holds at once, and what a round of them
// was measured to take: `base` + `fill` (epilogue, of a full round) + `step` per
// step of K, at least `least`; microseconds, for one and two parts per value.
// 256: 8 waves of 128 x 64, 128: 4 of 64 x 64, 64: 4 of 32 x 32.  (8 waves of
// 64 x 64 on 256 x 128 with three buffers were never the best.)  Steps on the
// 1,024 to 4,096-wide products: 256 x 256 tiles are best from about 2,048 on,
// 64 x 64 up to about 512: 8 matrices of 1,024 with fp16 operands take 519, 387
// and 559 us, 2 of them 411, 304 and 218, one of 4,096 1,782, 1,843 and 2,100.
struct Tile {
  int side, slots;
  double base, fill[2], step[2], least[2];
};
constexpr Tile kTiles[] = {{256, 256, 10, {27, 36}, {1.53, 2.37}, {0.95, 1.4}},
                           {128, 512, 6, {4, 12}, {1.12, 1.3}, {0.6, 0.9}},
                           {64, 512, 3, {1, 1}, {0.65, 0.65}, {0.45, 0.46}}};

struct Choice {
  int tile = -1;   // of kTiles
  Sched s;
  size_t part_bytes() const {
    const size_t side = kTiles[tile].side;
    return s.ragged ? up256(static_cast<size_t>(s.ragged) * s.slices * side * side * 4) : 0;
  }
};

struct Plan {
  int64_t G, m, n, mp, np;    // smaller and larger side, padded
  int parts;                  // per value
  int pad;                    // 256, 128 or 64: both sides are padded to it, tiles are at most it
  bool flip;                  // rows > cols
  size_t norm, x, a;          // bytes: norm partials, one X (or X^T), one A (or B)
  size_t part;                // partial tiles
  int slabs;                  // small_kernel's, 0: products of tiles
  Choice gram, poly, step;
  size_t total() const { return slabs ? norm + x + 2 * a : norm + 4 * x + 2 * a + part; }
};

// Tile and K cuts of one product, the quickest by these figures; a join takes 5 us
// and its parts' traffic twice.
Choice choose(const Plan& p, int64_t M, int64_t N, int64_t K, bool sym) {
  Choice best;
  double best_us = 0;
  for (int i = 0; i < 3; ++i) {
    const Tile& t = kTiles[i];
    if (t.side > p.pad) continue;
    const int64_t tm = M / t.side, tn = N / t.side;
    Sched s{};
    s.tiles_m = static_cast<int>(tm);
    s.tiles_n = static_cast<int>(tn);
    s.tiles = static_cast<int>(sym ? tm * (tm + 1) / 2 : tm * tn);
    s.steps = static_cast<int>(K * p.parts / 64);
    const int64_t all = s.tiles * p.G, rounds = all / t.slots, left = all - rounds * t.slots;
    const double step = t.step[p.parts - 1], least = t.least[p.parts - 1], fill = t.fill[p.parts - 1];
    for (int slices : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32}) {
      if (slices > 1 && (left == 0 || s.steps / slices < 4 || left * slices > t.slots)) continue;
      s.len = (s.steps + slices - 1) / slices;
      s.slices = (s.steps + s.len - 1) / s.len;
      s.whole = slices == 1 ? all : all - left;
      s.ragged = all - s.whole;
      const double part = static_cast<double>(left * s.slices) / t.slots;   // of the card, in the last round
      double us = rounds * (t.base + fill + s.steps * step);
      if (left) us += t.base + fill * part + s.len * std::max(least, step * part);
      if (slices > 1) us += 5.0 + 2 * left * s.slices * (t.side * t.side * 4.0) / 8e6;
      if (best.tile < 0 || us < best_us) {
        best.tile = i;
        best.s = s;
        best_us = us;
      }
    }
  }
  return best;
}

// Columns up to which slabs are used (each launch reads every slab's part of A).
// Measured against products of tiles, us: 64 x 64 25 and 69, 64 x 602 52 and 94,
// 64 x 8,192 89 and 147, 128 x 128 58 and 83 with fp32 products; 15 and 58, 40 and 79,
// 77 and 132, 31 and 69 with fp16 operands.  Of more than 64 rows and 128 columns: with fp32
// products 93 and 91 (128 x 256), 202 and 165 (128 x 8,192), an update of 128 x 1,433 134
// and 115; with fp16 operands 62 and 74, 170 and 144, 82 and 96 (128 x 1,433).
int64_t small_most(int64_t m, int parts) { return m <= 64 ? 8192 : m > 128 ? 0 : parts == 1 ? 2048 : kSlab; }

Plan plan(const gist_muon_desc* D) {
  Plan p{};
  p.G = D->groups > 1 ? D->groups : 1;
  p.flip = D->rows > D->cols;
  p.m = std::min(D->rows, D->cols);
  p.n = std::max(D->rows, D->cols);
  p.parts = D->dtype == GIST_DTYPE_F32 ? 2 : 1;
  p.norm = up256(static_cast<size_t>(p.G) * kNormBlocks * sizeof(double));
  p.slabs = p.n <= small_most(p.m, p.parts) ? static_cast<int>((p.n + kSlab - 1) / kSlab) : 0;
  if (p.slabs) {   // the slabs, and A's parts of two launches
    const size_t mp = p.m <= 64 ? 64 : 128, low = p.m <= 64 ? 3 : 10;
    p.x = up256(static_cast<size_t>(p.G) * p.slabs * kSlab * mp * p.parts * 2);
    p.a = up256(static_cast<size_t>(p.G) * p.slabs * low * 4096);
    return p;
  }
  // Larger padding allows larger tiles; it is taken where there are a few of
  // them and it adds at most 15% to the matrix.
  for (p.pad = 256; p.pad > 64; p.pad /= 2) {
    const int64_t a = (p.m + p.pad - 1) / p.pad * p.pad, b = (p.n + p.pad - 1) / p.pad * p.pad;
    if (p.m >= 4 * p.pad && 100 * a * b <= 115 * p.m * p.n) break;
  }
  p.mp = (p.m + p.pad - 1) / p.pad * p.pad;
  p.np = (p.n + p.pad - 1) / p.pad * p.pad;
  p.x = up256(static_cast<size_t>(p.G) * p.parts * p.mp * p.np * 2);
  p.a = up256(static_cast<size_t>(p.G) * p.parts * p.mp * p.mp * 2);
  p.part = 0;
  p.gram = choose(p, p.mp, p.mp, p.np, true);
  p.poly = choose(p, p.mp, p.mp, p.mp, true);
  p.step = choose(p, p.mp, p.np, p.mp, false);
  for (const Choice* c : {&p.gram, &p.poly, &p.step}) p.part = std::max(p.part, c->part_bytes());
  return p;
}

template <int NP, int MODE>
void product(hipStream_t st, const Plan& p, int64_t M, int64_t N, int64_t K, const Mat& P, const Mat& Q,
             const Epi& E, float* part) {
  static const char* const names[4] = {"muon_gram", "muon_poly", "muon_step", "muon_last"};
  constexpr bool kSym = MODE == kGram || MODE == kPoly;
  const Choice& c = MODE == kGram ? p.gram : MODE == kPoly ? p.poly : p.step;
  {
    ProfScope ps(st, names[MODE], (kSym ? 1.0 : 2.0) * p.G * M * N * K, 2.0 * NP * p.G * (M * K + N * K + M * N));
    const dim3 g(static_cast<unsigned>(c.s.whole + c.s.ragged * c.s.slices));
    if (c.tile == 0) product_kernel<NP, MODE, 4, 2, 2, 4, 2><<<g, 512, 0, st>>>(c.s, P, Q, E, part);
    else if (c.tile == 1) product_kernel<NP, MODE, 2, 2, 2, 2, 2><<<g, 256, 0, st>>>(c.s, P, Q, E, part);
    else product_kernel<NP, MODE, 1, 1, 2, 2, 4><<<g, 256, 0, st>>>(c.s, P, Q, E, part);
  }
  if (c.s.ragged) {
    ProfScope ps(st, "muon_join", 0.0, static_cast<double>(c.part_bytes()));
    const int nb = kTiles[c.tile].side / 32;
    const dim3 g(static_cast<unsigned>((c.s.ragged * nb * nb + 3) / 4));
    if (c.tile == 0) join_kernel<NP, MODE, 256><<<g, kBlock, 0, st>>>(c.s, part, E);
    else if (c.tile == 1) join_kernel<NP, MODE, 128><<<g, kBlock, 0, st>>>(c.s, part, E);
    else join_kernel<NP, MODE, 64><<<g, kBlock, 0, st>>>(c.s, part, E);
  }
}

dim3 norm_grid(int64_t count, int64_t G) {
  return dim3(static_cast<unsigned>(std::min<int64_t>(kNormBlocks, (count + 8 * kBlock - 1) / (8 * kBlock))),
              static_cast<unsigned>(G));
}

void launch_norm(hipStream_t st, const Plan& p, int64_t count, const float* G, float* M, bool update, bool vec,
                 const Update& u, double* part) {
  ProfScope ps(st, "muon_norm", 4.0 * p.G * count, (update ? 12.0 : 4.0) * p.G * count);
  const dim3 g = norm_grid(count, p.G);
  if (update && vec) norm_kernel<true, 4><<<g, kBlock, 0, st>>>(count, G, M, u, part);
  else if (update) norm_kernel<true, 1><<<g, kBlock, 0, st>>>(count, G, M, u, part);
  else if (vec) norm_kernel<false, 4><<<g, kBlock, 0, st>>>(count, G, M, u, part);
  else norm_kernel<false, 1><<<g, kBlock, 0, st>>>(count, G, M, u, part);
}

template <int NP>
gist_status run_small(hipStream_t st, const gist_muon_desc* D, const Plan& p, const float* G, void* O, float* W,
                      float* M, const Update& u, bool vec, char* ws) {
  const int64_t count = D->rows * D->cols;
  SmallArgs a{};
  a.rows = D->rows;
  a.cols = D->cols;
  a.m = static_cast<int>(p.m);
  a.n = static_cast<int>(p.n);
  a.slabs = p.slabs;
  a.flip = p.flip;
  a.G = G;
  a.M = M;
  a.W = W;
  a.O = O;
  a.u = u;
  a.norm = reinterpret_cast<const double*>(ws);
  a.eps = D->eps;
  a.ca = D->coef[0];
  a.cb = D->coef[1];
  a.cc = D->coef[2];
  a.steps = D->steps;
  a.T = ws + p.norm;
  float* const parts[2] = {reinterpret_cast<float*>(ws + p.norm + p.x),
                           reinterpret_cast<float*>(ws + p.norm + p.x + p.a)};
  if (p.slabs > 1) {
    launch_norm(st, p, count, G, M, W != nullptr, vec, u, reinterpret_cast<double*>(ws));
    a.nparts = static_cast<int>(norm_grid(count, p.G).x);
  }
  // one slab takes every step in one launch; several a launch for A's first parts and
  // one for each step
  for (int k = p.slabs > 1 ? -1 : 0; k < (p.slabs > 1 ? D->steps : 1); ++k) {
    a.first = p.slabs == 1 || k < 0;
    a.k0 = std::max(k, 0);
    a.k1 = p.slabs == 1 ? D->steps : k + 1;
    a.pin = parts[k & 1];
    a.pout = parts[(k & 1) ^ 1];
    ProfScope ps(st, "muon_small", 0.0, 0.0);
    const dim3 g(static_cast<unsigned>(p.slabs), static_cast<unsigned>(p.G));
#define SMALL(MP)                                                                      \
  do {                                                                                 \
    if (W) small_kernel<NP, MP, true><<<g, kSmallThreads, 0, st>>>(a);                 \
    else small_kernel<NP, MP, false><<<g, kSmallThreads, 0, st>>>(a);                  \
  } while (0)
    if (p.m <= 64) SMALL(64);
    else SMALL(128);
#undef SMALL
  }
  return check_launch("muon");
}

template <int NP>
gist_status run(hipStream_t st, const gist_muon_desc* D, const float* G, void* O, float* W,
                float* M, Update u, char* ws) {
  const Plan p = plan(D);
  const int64_t count = D->rows * D->cols;
  const bool vec = D->cols % 4 == 0 && reinterpret_cast<uintptr_t>(G) % 16 == 0 &&
                   (!W || reinterpret_cast<uintptr_t>(M) % 16 == 0);
  if (p.slabs) return run_small<NP>(st, D, p, G, O, W, M, u, vec, ws);
  double* part = reinterpret_cast<double*>(ws);
  ws += p.norm;
  auto mat = [&](size_t bytes, int64_t r, int64_t c) {
    Mat x{reinterpret_cast<_Float16*>(ws), c, NP * r * c};
    ws += bytes;
    return x;
  };
  Mat X[2], T[2];
  for (int i = 0; i < 2; ++i) {
    X[i] = mat(p.x, p.mp, p.np);
    T[i] = mat(p.x, p.np, p.mp);
  }
  const Mat A = mat(p.a, p.mp, p.mp), B = mat(p.a, p.mp, p.mp);
  float* parts = reinterpret_cast<float*>(ws);
  const int nb = static_cast<int>(norm_grid(count, p.G).x);
  launch_norm(st, p, count, G, M, W != nullptr, vec, u, part);
  {
    ProfScope ps(st, "muon_split", 0.0, (4.0 * (W ? 2 : 1) + 4.0 * NP) * p.G * count);
    const int64_t rp = p.flip ? p.np : p.mp, cp = p.flip ? p.mp : p.np;
    const dim3 g(static_cast<unsigned>(cp / 64), static_cast<unsigned>(rp / 64), static_cast<unsigned>(p.G));
    const Mat& d = p.flip ? T[0] : X[0];
    const Mat& tr = p.flip ? X[0] : T[0];
#define SPLIT(U, V) split_kernel<U, NP, V><<<g, kBlock, 0, st>>>(D->rows, D->cols, nb, G, M, u, part, D->eps, d, tr)
    if (W && vec) SPLIT(true, true);
    else if (W) SPLIT(true, false);
    else if (vec) SPLIT(false, true);
    else SPLIT(false, false);
#undef SPLIT
  }
  int cur = 0;
  for (int k = 0; k < D->steps; ++k) {
    Epi e{};
    e.out = A;
    product<NP, kGram>(st, p, p.mp, p.mp, p.np, X[cur], X[cur], e, parts);
    e.out = B;
    e.add = A;
    e.alpha = D->coef[1];
    e.beta = D->coef[2];
    product<NP, kPoly>(st, p, p.mp, p.mp, p.mp, A, A, e, parts);
    e.add = X[cur];
    e.alpha = D->coef[0];
    e.beta = 1.f;
    if (k + 1 < D->steps) {
      e.out = X[cur ^ 1];
      e.outT = T[cur ^ 1];
      product<NP, kStep>(st, p, p.mp, p.np, p.mp, B, T[cur], e, parts);
      cur ^= 1;
    } else {
      e.W = W;
      e.O = O;
      e.m = p.m;
      e.n = p.n;
      e.si = p.flip ? 1 : D->cols;
      e.sj = p.flip ? D->cols : 1;
      e.group = count;
      e.keep = u.keep;
      e.eta = u.eta;
      e.o_half = NP == 1;
      // every group and row begins at a multiple of eight elements
      e.vec = D->cols % 8 == 0 && reinterpret_cast<uintptr_t>(W ? static_cast<void*>(W) : O) % 16 == 0;
      product<NP, kLast>(st, p, p.mp, p.np, p.mp, B, T[cur], e, parts);
    }
  }
  return check_launch("muon");
}

}  // namespace

size_t muon_workspace(const gist_muon_desc* D) { return plan(D).total(); }

gist_status muon(hipStream_t st, const gist_muon_desc* D, const float* G, void* O, float* W,
                 float* M, float lr, float momentum, float decay, float scale, void* ws) {
  Update u;
  u.momentum = momentum;
  u.omu = static_cast<float>(1.0 - static_cast<double>(momentum));
  u.keep = static_cast<float>(1.0 - static_cast<double>(lr) * decay);
  u.eta = static_cast<float>(static_cast<double>(lr) * scale);
  u.nesterov = (D->flags & GIST_MUON_NESTEROV) != 0;
  u.fresh = (D->flags & GIST_MUON_FRESH) != 0;
  char* w = static_cast<char*>(ws);
  return D->dtype == GIST_DTYPE_F32 ? run<2>(st, D, G, O, W, M, u, w) : run<1>(st, D, G, O, W, M, u, w);
}

}  // namespace gist
