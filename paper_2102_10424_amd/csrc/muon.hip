// Orthogonalised updates: X = U / max(||U||_F, eps), then Newton-Schulz steps
//   A = X X^T,  B = b A + c A A,  X <- a X + B X
// on the fp16 matrix cores, and the weight update along the result.
//
// Operands.  |entries| <= singular values <= 8 (checked by the caller), so
// matrices are held times S = 2^12: fp16 then keeps 11 significant bits of
// entries from 2^-26 up, and all that is below 2^-37 is lost.  fp32 products hold
// every value in two parts, hi = fp16(v), lo = fp16(v - hi) (22 to 23 bits, a
// float has 24) and take three products, hi hi' + hi lo' + lo hi'; lo lo' is
// below 2^-24 of the product.  With fp16 operands there is the one part.
// The parts are written by the kernel that produces a matrix, so the products
// load them as they are.  Matrices are padded with zeros to whole tiles, so
// that no product has edges: zero rows and columns stay zero.
//
// All three products are row times row (K contiguous in both operands): A and
// B are symmetric, and X is kept both as X (m x n) and as X^T (n x m), m <= n.

#include <algorithm>

#include "elem.cuh"

namespace gist {

namespace {

constexpr int kBlock = 256;
constexpr float kS = 4096.f, kInvS = 1.f / 4096.f;
constexpr int kPad = 64;        // padding of both sides
constexpr int kNormBlocks = 256;

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
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

// The new momentum, and per block the sum of squares of the direction, in
// double: part[group * kNormBlocks + block].
template <bool UPDATE>
__global__ __launch_bounds__(kBlock) void norm_kernel(int64_t count, const float* __restrict__ G,
                                                      float* __restrict__ M, Update u,
                                                      double* __restrict__ part) {
  __shared__ double sh[kBlock];
  const int64_t off = blockIdx.y * count;
  double s = 0.0;
  for (int64_t e = blockIdx.x * static_cast<int64_t>(kBlock) + threadIdx.x; e < count;
       e += static_cast<int64_t>(gridDim.x) * kBlock) {
    float v = G[off + e];
    if constexpr (UPDATE) {
      const float old = u.fresh ? 0.f : M[off + e];
      const float m = fmaf(u.momentum, old, u.omu * v);
      M[off + e] = m;
      v = direction(u, v, m);
    }
    s += static_cast<double>(v) * v;
  }
  sh[threadIdx.x] = s;
  __syncthreads();
  for (int o = kBlock / 2; o > 0; o >>= 1) {
    if (threadIdx.x < o) sh[threadIdx.x] += sh[threadIdx.x + o];
    __syncthreads();
  }
  if (threadIdx.x == 0) part[blockIdx.y * kNormBlocks + blockIdx.x] = sh[0];
}

template <int NP>
__device__ __forceinline__ void parts_of(float v, _Float16 (&p)[NP]) {
  p[0] = static_cast<_Float16>(v);
  if constexpr (NP == 2) p[1] = static_cast<_Float16>(v - static_cast<float>(p[0]));
}

// A matrix's parts: part p of element (i, j) at p * plane + i * ld + j.
struct Mat {
  _Float16* p;
  int64_t ld, plane, group;
};

// U / norm, split, as it stands (D) and transposed (T); 64 x 64 tiles over the
// padded sides.
template <bool UPDATE, int NP>
__global__ __launch_bounds__(kBlock) void split_kernel(int64_t rows, int64_t cols, int nparts,
                                                       const float* __restrict__ G,
                                                       const float* __restrict__ M, Update u,
                                                       const double* __restrict__ part, float eps,
                                                       Mat D, Mat T) {
  __shared__ double red[kBlock];
  __shared__ float tile[64][65];
  const int t = threadIdx.x;
  const int64_t g = blockIdx.z, off = g * rows * cols;
  red[t] = t < nparts ? part[g * kNormBlocks + t] : 0.0;
  __syncthreads();
  for (int o = kBlock / 2; o > 0; o >>= 1) {
    if (t < o) red[t] += red[t + o];
    __syncthreads();
  }
  // a norm past fp32 (entries beyond 10^30): both scaled down
  double norm = sqrt(red[0]);
  const bool huge = norm > 1e30;
  const float pre = huge ? 0x1p-64f : 1.f;
  if (huge) norm *= 0x1p-64;
  const float div = norm < static_cast<double>(eps) ? eps : static_cast<float>(norm);   // NaN stays
  const int64_t r0 = blockIdx.y * 64, c0 = blockIdx.x * 64;
  _Float16* const d = D.p + g * D.group;
  _Float16* const tr = T.p + g * T.group;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int r = i * 4 + (t >> 6), c = t & 63;
    float v = 0.f;
    if (r0 + r < rows && c0 + c < cols) {
      const int64_t e = off + (r0 + r) * cols + c0 + c;
      v = G[e];
      if constexpr (UPDATE) v = direction(u, v, M[e]);
      v = kS * (v * pre / div);
    }
    tile[r][c] = v;
    _Float16 p[NP];
    parts_of<NP>(v, p);
#pragma unroll
    for (int q = 0; q < NP; ++q) d[q * D.plane + (r0 + r) * D.ld + c0 + c] = p[q];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int c = i * 4 + (t >> 6), r = t & 63;
    _Float16 p[NP];
    parts_of<NP>(tile[r][c], p);
#pragma unroll
    for (int q = 0; q < NP; ++q) tr[q * T.plane + (c0 + c) * T.ld + r0 + r] = p[q];
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
};

template <int NP>
__device__ __forceinline__ float value_of(const Mat& a, int64_t g, int64_t i, int64_t j) {
  const _Float16* p = a.p + g * a.group + i * a.ld + j;
  float v = static_cast<float>(p[0]);
  if constexpr (NP == 2) v += static_cast<float>(p[a.plane]);
  return v;
}

// P Q^T (rows of both K contiguous): 64 x 64 tiles, a 32 x 32 block per wave,
// fragments straight from memory.
template <int NP, int MODE>
__global__ __launch_bounds__(kBlock) void product_kernel(int64_t K, Mat P, Mat Q, Epi E) {
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int li = lane & 31, lh = lane >> 5;
  const int64_t g = blockIdx.z;
  const int64_t i0 = blockIdx.y * 64 + (wave >> 1) * 32, j0 = blockIdx.x * 64 + (wave & 1) * 32;
  const _Float16* p = P.p + g * P.group + (i0 + li) * P.ld + 8 * lh;
  const _Float16* q = Q.p + g * Q.group + (j0 + li) * Q.ld + 8 * lh;
  floatx16 acc = {};
  for (int64_t k = 0; k < K; k += 16) {
    half8 a[NP], b[NP];
#pragma unroll
    for (int s = 0; s < NP; ++s) {
      a[s] = *reinterpret_cast<const half8*>(p + s * P.plane + k);
      b[s] = *reinterpret_cast<const half8*>(q + s * Q.plane + k);
    }
    if constexpr (NP == 2) {
      acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[0], b[1], acc, 0, 0, 0);
      acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[1], b[0], acc, 0, 0, 0);
    }
    acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[0], b[0], acc, 0, 0, 0);
  }
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int64_t i = i0 + 8 * (r >> 2) + 4 * lh + (r & 3), j = j0 + li;
    float v = acc[r] * kInvS;   // the product times S
    if constexpr (MODE != kGram) v = fmaf(E.alpha, value_of<NP>(E.add, g, i, j), E.beta * v);
    if constexpr (MODE == kLast) {
      if (i >= E.m || j >= E.n) continue;
      const int64_t e = g * E.group + i * E.si + j * E.sj;
      v *= kInvS;
      if (E.W) E.W[e] = fmaf(-E.eta, v, E.keep * E.W[e]);
      else if (E.o_half) static_cast<_Float16*>(E.O)[e] = static_cast<_Float16>(v);
      else static_cast<float*>(E.O)[e] = v;
    } else {
      _Float16 s[NP];
      parts_of<NP>(v, s);
#pragma unroll
      for (int x = 0; x < NP; ++x) {
        E.out.p[g * E.out.group + x * E.out.plane + i * E.out.ld + j] = s[x];
        if constexpr (MODE == kStep)
          E.outT.p[g * E.outT.group + x * E.outT.plane + j * E.outT.ld + i] = s[x];
      }
    }
  }
}

size_t up256(size_t x) { return (x + 255) & ~size_t(255); }

struct Plan {
  int64_t G, m, n, mp, np;    // smaller and larger side, padded
  int parts;                  // per value
  bool flip;                  // rows > cols
  size_t norm, x, a;          // bytes: norm partials, one X (or X^T), one A (or B)
  size_t total() const { return norm + 4 * x + 2 * a; }
};

Plan plan(const gist_muon_desc* D) {
  Plan p;
  p.G = D->groups > 1 ? D->groups : 1;
  p.flip = D->rows > D->cols;
  p.m = std::min(D->rows, D->cols);
  p.n = std::max(D->rows, D->cols);
  p.mp = (p.m + kPad - 1) / kPad * kPad;
  p.np = (p.n + kPad - 1) / kPad * kPad;
  p.parts = D->dtype == GIST_DTYPE_F32 ? 2 : 1;
  p.norm = up256(static_cast<size_t>(p.G) * kNormBlocks * sizeof(double));
  p.x = up256(static_cast<size_t>(p.G) * p.parts * p.mp * p.np * 2);
  p.a = up256(static_cast<size_t>(p.G) * p.parts * p.mp * p.mp * 2);
  return p;
}

template <int NP, int MODE>
void product(hipStream_t st, int64_t M, int64_t N, int64_t K, int64_t G, const Mat& P, const Mat& Q,
             const Epi& E) {
  static const char* const names[4] = {"muon_gram", "muon_poly", "muon_step", "muon_last"};
  ProfScope ps(st, names[MODE], 2.0 * G * M * N * K, 2.0 * NP * G * (M * K + N * K + M * N));
  const dim3 g(static_cast<unsigned>(N / kPad), static_cast<unsigned>(M / kPad), static_cast<unsigned>(G));
  product_kernel<NP, MODE><<<g, kBlock, 0, st>>>(K, P, Q, E);
}

template <int NP>
gist_status run(hipStream_t st, const gist_muon_desc* D, const float* G, void* O, float* W,
                float* M, Update u, char* ws) {
  const Plan p = plan(D);
  const int64_t count = D->rows * D->cols;
  double* part = reinterpret_cast<double*>(ws);
  ws += p.norm;
  auto mat = [&](size_t bytes, int64_t r, int64_t c) {
    Mat x{reinterpret_cast<_Float16*>(ws), c, r * c, NP * r * c};
    ws += bytes;
    return x;
  };
  Mat X[2], T[2];
  for (int i = 0; i < 2; ++i) {
    X[i] = mat(p.x, p.mp, p.np);
    T[i] = mat(p.x, p.np, p.mp);
  }
  const Mat A = mat(p.a, p.mp, p.mp), B = mat(p.a, p.mp, p.mp);
  const int nb = static_cast<int>(std::min<int64_t>(kNormBlocks, (count + kBlock - 1) / kBlock));
  {
    ProfScope ps(st, "muon_norm", 4.0 * p.G * count, (W ? 12.0 : 4.0) * p.G * count);
    const dim3 g(nb, static_cast<unsigned>(p.G));
    if (W) norm_kernel<true><<<g, kBlock, 0, st>>>(count, G, M, u, part);
    else norm_kernel<false><<<g, kBlock, 0, st>>>(count, G, M, u, part);
  }
  {
    ProfScope ps(st, "muon_split", 0.0, (4.0 * (W ? 2 : 1) + 4.0 * NP) * p.G * count);
    const int64_t rp = p.flip ? p.np : p.mp, cp = p.flip ? p.mp : p.np;
    const dim3 g(static_cast<unsigned>(cp / 64), static_cast<unsigned>(rp / 64), static_cast<unsigned>(p.G));
    const Mat& d = p.flip ? T[0] : X[0];
    const Mat& tr = p.flip ? X[0] : T[0];
    if (W) split_kernel<true, NP><<<g, kBlock, 0, st>>>(D->rows, D->cols, nb, G, M, u, part, D->eps, d, tr);
    else split_kernel<false, NP><<<g, kBlock, 0, st>>>(D->rows, D->cols, nb, G, M, u, part, D->eps, d, tr);
  }
  int cur = 0;
  for (int k = 0; k < D->steps; ++k) {
    Epi e{};
    e.out = A;
    product<NP, kGram>(st, p.mp, p.mp, p.np, p.G, X[cur], X[cur], e);
    e.out = B;
    e.add = A;
    e.alpha = D->coef[1];
    e.beta = D->coef[2];
    product<NP, kPoly>(st, p.mp, p.mp, p.mp, p.G, A, A, e);
    e.add = X[cur];
    e.alpha = D->coef[0];
    e.beta = 1.f;
    if (k + 1 < D->steps) {
      e.out = X[cur ^ 1];
      e.outT = T[cur ^ 1];
      product<NP, kStep>(st, p.mp, p.np, p.mp, p.G, B, T[cur], e);
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
      product<NP, kLast>(st, p.mp, p.np, p.mp, p.G, B, T[cur], e);
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
