// Log probabilities of given classes, entropy, log-sum-exp and the K best
// classes of every row of logits, and the gradient of the first two.
//
// One pass over a row.  With L = log2 e and m the largest logit so far, a
// thread keeps s = sum 2^y and t = sum y 2^y over its elements, y = (z - m) L;
// a larger m' rescales both,
//   s <- c s,  t <- c (t + D s),  D = (m - m') L,  c = 2^D.
// At the end lse = m + log2(s) / L and entropy = (log2 s - t / s) / L.  y is
// clamped from below at -300, where 2^y is 0: a masked (-Inf) logit, or one whose
// distance to m overflows, then adds 0 instead of 0 * Inf.  (One fma, z L - m L,
// would do for y, but m L overflows in a row of the type's lowest value.)
//
// The K best are kept by each wave as 64 sorted integers, one per lane: the
// logit's bits in an order-keeping form above the inverted class, so that one
// unsigned comparison orders by value and then by ascending class.  Most
// elements fail the comparison with the K-th and cost no more than that.

#include <algorithm>

#include "elem.cuh"

namespace gist {

namespace {

constexpr int kBlock = 256;
constexpr int kWaves = kBlock / 64;
constexpr float kL = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kFloor = -300.f;

typedef unsigned long long u64;

__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float lg2(float x) { return __builtin_amdgcn_logf(x); }
// The larger, or NaN if either is one (fmaxf would drop it).
__device__ __forceinline__ float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }

struct Stat {
  float m, s, t;
};

__device__ __forceinline__ void rescale(Stat& a, float m) {
  const float D = fmaxf((a.m - m) * kL, kFloor);
  const float c = ex2(D);
  a.t = c * fmaf(D, a.s, a.t);
  a.s *= c;
  a.m = m;
}

__device__ __forceinline__ void merge(Stat& a, Stat b) {
  const float m = max_nan(a.m, b.m);
  rescale(a, m);
  rescale(b, m);
  a.s += b.s;
  a.t += b.t;
}

__device__ __forceinline__ Stat wave_merge(Stat a) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1)
    merge(a, Stat{__shfl_xor(a.m, o, 64), __shfl_xor(a.s, o, 64), __shfl_xor(a.t, o, 64)});
  return a;
}

// Logit and class in one integer, greater for a greater logit or an equal
// one of a lower class; 0 is below all.
__device__ __forceinline__ unsigned order_bits(float z) {
  const int u = __float_as_int(z + 0.f);   // -0 equals 0
  return static_cast<unsigned>(u) ^ (static_cast<unsigned>(u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float from_order(unsigned k) {
  return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
__device__ __forceinline__ u64 pack(float z, unsigned cls) {
  return (static_cast<u64>(order_bits(z)) << 32) | (0xffffffffu - cls);
}

// A wave's sorted list, lane l holding the l-th best; thr is the K-th.
struct Top {
  u64 mine = 0, thr = 0;
  int K;
  // Candidates of all lanes (0: none).
  __device__ __forceinline__ void offer(u64 x, int lane) {
    u64 want = __ballot(x > thr);
    while (want) {
      const int src = __ffsll(want) - 1;
      want &= want - 1;
      const u64 c = __shfl(x, src, 64);
      if (c <= thr) continue;
      const int at = __popcll(__ballot(mine > c));
      const u64 up = __shfl_up(mine, 1, 64);
      mine = lane < at ? mine : lane == at ? c : up;
      thr = __shfl(mine, K - 1, 64);
    }
  }
};

struct Out {
  const int* tokens;
  float *logp, *entropy, *lse, *top;
  int* idx;
};

// A row's outputs from its statistics; called by one wave.
template <int STORE>
__device__ __forceinline__ void write_row(const Out& o, int64_t row, int C, const void* Z,
                                          int64_t ldz, Stat a, const Top& top, int K, int lane) {
  const float nan = __uint_as_float(0x7fc00000u);
  const bool ok = a.m < INFINITY;            // no NaN, no +Inf in the row
  const bool some = ok && a.m > -INFINITY;   // not masked throughout
  const float l2 = lg2(a.s);
  const float lse = some ? fmaf(kLn2, l2, a.m) : ok ? -INFINITY : nan;
  if (lane == 0) {
    if (o.lse) o.lse[row] = lse;
    if (o.entropy) o.entropy[row] = some ? kLn2 * (l2 - a.t / a.s) : ok ? 0.f : nan;
    if (o.logp) {
      const int y = o.tokens[row];
      float v = 0.f;
      if (y >= C) {
        v = nan;
      } else if (y >= 0) {
        float z[1];
        load_vec<STORE, 1>(Z, row * ldz + y, z);
        v = z[0] == -INFINITY && ok ? -INFINITY : z[0] - lse;
      }
      o.logp[row] = ok ? v : nan;
    }
  }
  if (lane < K) {
    const float z = from_order(static_cast<unsigned>(top.mine >> 32));
    o.top[row * K + lane] = !ok ? nan : z == -INFINITY ? z : z - lse;
    o.idx[row * K + lane] = ok ? static_cast<int>(0xffffffffu - static_cast<unsigned>(top.mine)) : -1;
  }
}

// One workgroup per (row, part of the row).  parts == 1 writes the outputs,
// else the part's statistics (4 floats) and list (K integers) go to `part`.
template <int STORE, int V, bool TOP>
__global__ __launch_bounds__(kBlock) void rows_kernel(int64_t items, int parts, int64_t len, int C,
                                                      const void* __restrict__ Z, int64_t ldz,
                                                      Out o, int K, float* __restrict__ pstat,
                                                      u64* __restrict__ ptop) {
  __shared__ Stat wst[kWaves];
  __shared__ u64 wtop[kWaves][64];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int64_t row = parts == 1 ? item : item / parts;
    const int64_t c0 = parts == 1 ? 0 : (item - row * parts) * len;
    const int64_t c1 = min<int64_t>(C, c0 + len);
    Stat a{-INFINITY, 0.f, 0.f};
    Top top;
    top.K = K;
    for (int64_t j0 = c0; j0 < c1; j0 += V * kBlock) {   // block-uniform: ballots inside
      const int64_t j = j0 + V * t;
      float z[V];
#pragma unroll
      for (int q = 0; q < V; ++q) z[q] = -INFINITY;
      const bool in = j < c1;   // widths are multiples of V
      if (in) load_vec<STORE, V>(Z, row * ldz + j, z);
      float m = z[0];
#pragma unroll
      for (int q = 1; q < V; ++q) m = max_nan(m, z[q]);
      if constexpr (TOP) {
        if (__any(in && pack(m, 0u) > top.thr)) {
#pragma unroll
          for (int q = 0; q < V; ++q)
            top.offer(in ? pack(z[q], static_cast<unsigned>(j + q)) : 0, lane);
        }
      }
      rescale(a, max_nan(a.m, m));
#pragma unroll
      for (int q = 0; q < V; ++q) {
        const float y = fmaxf((z[q] - a.m) * kL, kFloor);
        const float e = ex2(y);
        a.s += e;
        a.t = fmaf(e, y, a.t);
      }
    }
    a = wave_merge(a);
    __syncthreads();   // the previous item's LDS is read
    if (lane == 0) wst[wave] = a;
    if (TOP) wtop[wave][lane] = top.mine;
    __syncthreads();
    if (wave == 0) {
#pragma unroll
      for (int w = 1; w < kWaves; ++w) {
        merge(a, wst[w]);
        if (TOP) top.offer(lane < K ? wtop[w][lane] : 0, lane);
      }
      if (parts == 1) {
        write_row<STORE>(o, row, C, Z, ldz, a, top, TOP ? K : 0, lane);
      } else {
        if (lane == 0) {
          float* p = pstat + 4 * item;
          p[0] = a.m;
          p[1] = a.s;
          p[2] = a.t;
        }
        if (TOP && lane < K) ptop[item * K + lane] = top.mine;
      }
    }
  }
}

// Joins the parts of a row: one wave per row.
template <int STORE>
__global__ __launch_bounds__(64) void join_rows_kernel(int64_t n, int parts, int C,
                                                       const void* __restrict__ Z, int64_t ldz,
                                                       Out o, int K,
                                                       const float* __restrict__ pstat,
                                                       const u64* __restrict__ ptop) {
  const int lane = threadIdx.x;
  for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
    Stat a{-INFINITY, 0.f, 0.f};
    for (int p = lane; p < parts; p += 64) {
      const float* s = pstat + 4 * (row * parts + p);
      merge(a, Stat{s[0], s[1], s[2]});
    }
    a = wave_merge(a);
    Top top;
    top.K = K > 0 ? K : 1;
    for (int i = 0; i < parts * K; i += 64)
      top.offer(i + lane < parts * K ? ptop[row * parts * K + i + lane] : 0, lane);
    write_row<STORE>(o, row, C, Z, ldz, a, top, K, lane);
  }
}

// dz = g_l (1[j = y] - p) - g_H p (log p + H), p = exp(z - lse).  A group of
// 1 << tl threads per (row, slab of columns); with slabs the group is the block.
template <int STORE, int V>
__global__ __launch_bounds__(kBlock) void bwd_kernel(int64_t items, int slabs, int slab, int tl, int C,
                                                     const void* Z, int64_t ldz,
                                                     const int* __restrict__ tokens,
                                                     const float* __restrict__ lse,
                                                     const float* __restrict__ ent,
                                                     const float* __restrict__ gl,
                                                     const float* __restrict__ gh, void* dZ,
                                                     int64_t ldd) {
  const int lane = threadIdx.x & ((1 << tl) - 1);
  for (int64_t item = (static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x) >> tl; item < items;
       item += (static_cast<int64_t>(gridDim.x) * kBlock) >> tl) {
    const int64_t row = slabs == 1 ? item : item / slabs;
    const int64_t c0 = slabs == 1 ? 0 : (item - row * slabs) * slab;
    const int64_t c1 = min<int64_t>(C, c0 + slab);
    const float l = lse[row];
    const float a = gl ? gl[row] : 0.f, b = gh ? gh[row] : 0.f;
    const float h = gh ? ent[row] : 0.f;
    const int y = gl ? tokens[row] : -1;
    float gy = a;                            // weight of the given class's term
    float w0 = fmaf(b, h, y >= 0 ? a : 0.f), w1 = b;
    // a row without probabilities: 0; one with a NaN, or a token past the classes: NaN
    const bool none = l == -INFINITY;
    const bool bad = l != l || l == INFINITY || y >= C;
    if (none) gy = 0.f;
    for (int64_t j = c0 + V * lane; j < c1; j += V << tl) {
      float z[V], d[V];
      load_vec<STORE, V>(Z, row * ldz + j, z);
#pragma unroll
      for (int q = 0; q < V; ++q) {
        const float x = fmaxf(z[q] - l, -200.f);
        const float p = ex2(x * kL);
        d[q] = -p * fmaf(w1, x, w0);
        if (none) d[q] = 0.f;
        if (j + q == y) d[q] += gy;
        if (bad) d[q] = __uint_as_float(0x7fc00000u);
      }
      store_as<STORE, V>(dZ, row * ldd + j, d);
    }
  }
}

struct Plan {
  int v, parts;
  int64_t len;
};

// Parts of a row: as many as fill the card, of at least 4,096 elements each
// (16 per thread).
Plan plan_rows(int64_t n, int64_t C) {
  Plan p{1, 1, C};
  const int64_t want = n >= 1024 ? 1 : (1024 + n - 1) / std::max<int64_t>(n, 1);
  const int64_t most = C / 4096;
  p.parts = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({want, most, 256})));
  p.len = ((C + p.parts - 1) / p.parts + 7) / 8 * 8;
  p.parts = static_cast<int>((C + p.len - 1) / p.len);
  return p;
}

size_t up256(size_t x) { return (x + 255) & ~size_t(255); }

}  // namespace

size_t log_probs_workspace(int64_t n, int64_t C, int K) {
  const Plan p = plan_rows(n, C);
  if (p.parts == 1) return 0;
  return up256(static_cast<size_t>(n) * p.parts * 16) + static_cast<size_t>(n) * p.parts * K * 8;
}

gist_status log_probs(hipStream_t st, int64_t n, int64_t C, const void* Z, int64_t ldz, int store,
                      const int32_t* tokens, float* logp, float* entropy, float* lse, int K,
                      float* top_logp, int32_t* top_idx, void* ws) {
  const Plan p = plan_rows(n, C);
  const int eb = store == GIST_STORE_F32 ? 4 : 2;
  const int v = vec_of(store == GIST_STORE_F32 ? 4 : 8, C, ldz, Z, eb);
  const Out o{tokens, logp, entropy, lse, top_logp, top_idx};
  float* pstat = static_cast<float*>(ws);
  u64* ptop = p.parts == 1 ? nullptr
                           : reinterpret_cast<u64*>(static_cast<char*>(ws) +
                                                    up256(static_cast<size_t>(n) * p.parts * 16));
  const int64_t items = n * p.parts;
  const dim3 g(static_cast<unsigned>(std::min<int64_t>(items, 1 << 22)));
  {
    ProfScope ps(st, "log_probs", 6.0 * n * C, static_cast<double>(n) * C * eb);
#define ROWS1(S, W, T)                                                                         \
  rows_kernel<S, W, T><<<g, kBlock, 0, st>>>(items, p.parts, p.len, static_cast<int>(C), Z, ldz, o, \
                                             K, pstat, ptop)
#define ROWS(S, W)                     \
  do {                                 \
    if (K > 0) ROWS1(S, W, true);      \
    else ROWS1(S, W, false);           \
  } while (0)
    if (store == GIST_STORE_F32) {
      if (v == 4) ROWS(GIST_STORE_F32, 4);
      else if (v == 2) ROWS(GIST_STORE_F32, 2);
      else ROWS(GIST_STORE_F32, 1);
    } else if (store == GIST_STORE_BF16) {
      if (v == 8) ROWS(GIST_STORE_BF16, 8);
      else if (v == 4) ROWS(GIST_STORE_BF16, 4);
      else if (v == 2) ROWS(GIST_STORE_BF16, 2);
      else ROWS(GIST_STORE_BF16, 1);
    } else {
      if (v == 8) ROWS(GIST_STORE_F16, 8);
      else if (v == 4) ROWS(GIST_STORE_F16, 4);
      else if (v == 2) ROWS(GIST_STORE_F16, 2);
      else ROWS(GIST_STORE_F16, 1);
    }
#undef ROWS
#undef ROWS1
  }
  if (p.parts > 1) {
    ProfScope ps(st, "log_probs_join", 0.0, static_cast<double>(items) * (16 + 8 * K));
    const dim3 gj(static_cast<unsigned>(std::min<int64_t>(n, 1 << 22)));
    if (store == GIST_STORE_F32)
      join_rows_kernel<GIST_STORE_F32><<<gj, 64, 0, st>>>(n, p.parts, static_cast<int>(C), Z, ldz, o, K, pstat, ptop);
    else if (store == GIST_STORE_BF16)
      join_rows_kernel<GIST_STORE_BF16><<<gj, 64, 0, st>>>(n, p.parts, static_cast<int>(C), Z, ldz, o, K, pstat, ptop);
    else
      join_rows_kernel<GIST_STORE_F16><<<gj, 64, 0, st>>>(n, p.parts, static_cast<int>(C), Z, ldz, o, K, pstat, ptop);
  }
  return check_launch("log_probs");
}

gist_status log_probs_bwd(hipStream_t st, int64_t n, int64_t C, const void* Z, int64_t ldz,
                          int store, const int32_t* tokens, const float* lse,
                          const float* entropy, const float* g_logp, const float* g_entropy,
                          void* dZ, int64_t ldd) {
  const int eb = store == GIST_STORE_F32 ? 4 : 2, most = store == GIST_STORE_F32 ? 4 : 8;
  const int v = std::min(vec_of(most, C, ldz, Z, eb), vec_of(most, C, ldd, dZ, eb));
  const int tl = std::min(8, ceil_log2((C + v - 1) / v));
  // slabs of eight steps where a row takes more than one
  const int64_t step = static_cast<int64_t>(v) << tl;
  const int64_t slab = C <= 8 * step ? C : 8 * step;
  const int64_t slabs = (C + slab - 1) / slab, items = n * slabs;
  const dim3 g(static_cast<unsigned>(std::min<int64_t>(((items << tl) + kBlock - 1) / kBlock, 1 << 22)));
  ProfScope ps(st, "log_probs_bwd", 8.0 * n * C, 2.0 * n * C * eb);
#define BWD(S, W)                                                                                 \
  bwd_kernel<S, W><<<g, kBlock, 0, st>>>(items, static_cast<int>(slabs), static_cast<int>(slab), tl, \
                                         static_cast<int>(C), Z, ldz, tokens, lse, entropy, g_logp,  \
                                         g_entropy, dZ, ldd)
  if (store == GIST_STORE_F32) {
    if (v == 4) BWD(GIST_STORE_F32, 4);
    else if (v == 2) BWD(GIST_STORE_F32, 2);
    else BWD(GIST_STORE_F32, 1);
  } else if (store == GIST_STORE_BF16) {
    if (v == 8) BWD(GIST_STORE_BF16, 8);
    else if (v == 4) BWD(GIST_STORE_BF16, 4);
    else if (v == 2) BWD(GIST_STORE_BF16, 2);
    else BWD(GIST_STORE_BF16, 1);
  } else {
    if (v == 8) BWD(GIST_STORE_F16, 8);
    else if (v == 4) BWD(GIST_STORE_F16, 4);
    else if (v == 2) BWD(GIST_STORE_F16, 2);
    else BWD(GIST_STORE_F16, 1);
  }
#undef BWD
  return check_launch("log_probs_bwd");
}

}  // namespace gist
