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

__device__ __forceinline__ u64 lane_of(u64 x, int l) {   // l uniform
  const unsigned lo = __builtin_amdgcn_readlane(static_cast<unsigned>(x), l);
  const unsigned hi = __builtin_amdgcn_readlane(static_cast<unsigned>(x >> 32), l);
  return (static_cast<u64>(hi) << 32) | lo;
}
__device__ __forceinline__ u64 from_left(u64 x) {   // lane l - 1's
  const unsigned lo = __builtin_amdgcn_update_dpp(0, static_cast<int>(x), 0x138, 0xf, 0xf, false);
  const unsigned hi = __builtin_amdgcn_update_dpp(0, static_cast<int>(x >> 32), 0x138, 0xf, 0xf, false);
  return (static_cast<u64>(hi) << 32) | lo;
}

// A wave's sorted list, lane l holding the l-th best; thr is the K-th.
struct Top {
  u64 mine = 0, thr = 0;
  int K;
  __device__ __forceinline__ void exchange(int o, bool larger) {
    const u64 other = __shfl_xor(mine, o, 64);
    mine = (mine > other) == larger ? mine : other;
  }
  // Sorts any 64 integers, the greatest to lane 0.
  __device__ __forceinline__ void sort(u64 x, int lane) {
    mine = x;
#pragma unroll
    for (int size = 2; size <= 64; size <<= 1)
#pragma unroll
      for (int o = size >> 1; o > 0; o >>= 1) exchange(o, ((lane & o) == 0) == ((lane & size) == 0 || size == 64));
    thr = lane_of(mine, K - 1);
  }
  // Joins another sorted list, given in reverse (lane l holding its 63 - l-th).
  __device__ __forceinline__ void join(u64 reversed, int lane) {
    if (mine < reversed) mine = reversed;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) exchange(o, (lane & o) == 0);
    thr = lane_of(mine, K - 1);
  }
  // Candidates of all lanes (0: none), one insertion each.
  __device__ __forceinline__ void offer(u64 x, int lane) {
    u64 want = __ballot(x > thr);
    while (want) {
      const int src = __ffsll(want) - 1;
      want &= want - 1;
      const u64 c = lane_of(x, src);
      if (c <= thr) continue;
      const int at = __popcll(__ballot(mine > c));
      const u64 up = from_left(mine);
      mine = lane < at ? mine : lane == at ? c : up;
      thr = lane_of(mine, K - 1);
    }
  }
};

struct Out {
  const int* tokens;
  float *logp, *entropy, *lse, *top;
  int* idx;
};

// A row's outputs from its statistics, by one lane; returns log s = lse - m.  Log
// probabilities are (z - m) - log s, not z - lse: that keeps the bits of log s that lse
// loses to a large m (all of them in a row of the type's lowest value).
template <int STORE>
__device__ __forceinline__ float write_stats(const Out& o, int64_t row, int C, const void* Z, int64_t ldz,
                                             const Stat& a, bool write) {
  const float nan = __uint_as_float(0x7fc00000u);
  const bool ok = a.m < INFINITY;            // no NaN, no +Inf in the row
  const bool some = ok && a.m > -INFINITY;   // not masked throughout
  const float l2 = lg2(a.s);
  if (write) {
    if (o.lse) o.lse[row] = some ? fmaf(kLn2, l2, a.m) : ok ? -INFINITY : nan;
    if (o.entropy) o.entropy[row] = some ? kLn2 * (l2 - a.t / a.s) : ok ? 0.f : nan;
    if (o.logp) {
      const int y = o.tokens[row];
      float v = 0.f;
      if (y >= C) {
        v = nan;
      } else if (y >= 0) {
        float z[1];
        load_vec<STORE, 1>(Z, row * ldz + y, z);
        v = z[0] == -INFINITY && ok ? -INFINITY : (z[0] - a.m) - kLn2 * l2;
      }
      o.logp[row] = ok ? v : nan;
    }
  }
  return kLn2 * l2;
}

// The k-th best class (its order bits and itself) of a row.
__device__ __forceinline__ void write_top(const Out& o, int64_t row, int K, int k, unsigned bits, unsigned cls,
                                          float m, float ls) {
  const bool ok = m < INFINITY;
  const float z = from_order(bits);
  o.top[row * K + k] = !ok ? __uint_as_float(0x7fc00000u) : z == -INFINITY ? z : (z - m) - ls;
  o.idx[row * K + k] = ok ? static_cast<int>(cls) : -1;
}

// All of a row's outputs, by one wave.
template <int STORE>
__device__ __forceinline__ void write_row(const Out& o, int64_t row, int C, const void* Z, int64_t ldz,
                                          const Stat& a, const Top& top, int K, int lane) {
  const float ls = write_stats<STORE>(o, row, C, Z, ldz, a, lane == 0);
  if (lane < K)
    write_top(o, row, K, lane, static_cast<unsigned>(top.mine >> 32), 0xffffffffu - static_cast<unsigned>(top.mine),
              a.m, ls);
}

// ---- many short rows, one after another in memory: a lane a row ---------------

// 64 rows through LDS (an odd number of floats apart: lanes fall on different banks).  A
// lane walks its row twice, for the maximum and the K best, then for the sums.  The K best
// are a sorted list in registers: where v[k - 1] >= v[k], a logit's insertion leaves
// v[k] = the median of (z, v[k - 1], v[k]), one instruction; strictly greater logits alone
// move classes, so equal ones stay in order.  What bounds it: issue, 4 K + 12 instructions
// for 64 logits, and memory before it: 232,965 rows of 41 classes with the five best
// take 18 us; with lanes sharing a row (below), 21.
// When it is taken, us, here and there: 232,965 rows of 16 classes with the eight best 15.5
// and 18.4, of 24 with five 10.6 and 16.8; 100,000 of 40 with five 9.3 and 10.2, 60,000 of them
// 7.6 and 7.2, 1,536 6.3 and 4.8.  The most classes: 232,965 fp32 rows without any best take
// (43, 47, 56, 64 classes) 11.6, 12.6, 14.4, 16.2 and 9.7, 10.3, 11.4, 12.4, with five 18.3, 20.2,
// 24.9, 29.0 and 18.8, 19.0, 21.5, 21.5, with eight 24.9, 27.6, 32.8, 36.7 and 24.1, 24.1, 27.9,
// 27.9: the two meet at 42 or 43.  (A million rows with five: 56, 60, 76, 89 and 67, 67, 82, 86;
// the limit does not follow them up to where those meet, near 60.)
constexpr int kLaneClasses = 42, kLaneTop = 8;
constexpr int64_t kLaneRows = 98304;   // six waves a CU
template <int STORE, int K>
__global__ __launch_bounds__(64) void lane_rows_kernel(int64_t n, int C, unsigned inv, const void* __restrict__ Z,
                                                       Out o) {
  constexpr int V = STORE == GIST_STORE_F32 ? 4 : 8, kU = 4;
  extern __shared__ __attribute__((aligned(16))) float lds[];   // 64 rows of C | 1, and a vector
  const int lane = threadIdx.x, ld = C | 1;
  const int64_t r0 = static_cast<int64_t>(blockIdx.x) * 64;
  const int rows = static_cast<int>(min<int64_t>(64, n - r0)), count = rows * C;
  for (int e0 = V * lane; e0 < count; e0 += kU * 64 * V) {
    float x[kU][V];
#pragma unroll
    for (int u = 0; u < kU; ++u) load_some<STORE, V>(Z, r0 * C + e0 + u * 64 * V, count - e0 - u * 64 * V, 0.f, x[u]);
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int e = e0 + u * 64 * V;
      if (e >= count) break;
      if (C & 1) {
#pragma unroll
        for (int q = 0; q < V; q += 4)
          *reinterpret_cast<float4*>(lds + e + q) = float4{x[u][q], x[u][q + 1], x[u][q + 2], x[u][q + 3]};
      } else {
#pragma unroll
        for (int q = 0; q < V; q += 2) {   // a pair lies in one row; e / C by inv = 2^20 / C, rounded up
          const int at = e + q + static_cast<int>((static_cast<unsigned>(e + q) * inv) >> 20);
          lds[at] = x[u][q];
          lds[at + 1] = x[u][q + 1];
        }
      }
    }
  }
  __syncthreads();
  if (lane >= rows) return;
  const float* const z = lds + lane * ld;
  float m = -INFINITY, v[K > 0 ? K : 1];
  int cls[K > 0 ? K : 1];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    v[k] = -INFINITY;
    cls[k] = -1;
  }
#pragma unroll 8
  for (int j = 0; j < C; ++j) {
    const float x = z[j];
    m = max_nan(m, x);
    if constexpr (K > 0) {
      bool up[K];
#pragma unroll
      for (int k = 0; k < K; ++k) up[k] = x > v[k];
#pragma unroll
      for (int k = K - 1; k > 0; --k) {
        cls[k] = up[k - 1] ? cls[k - 1] : up[k] ? j : cls[k];
        v[k] = __builtin_amdgcn_fmed3f(x, v[k - 1], v[k]);
      }
      cls[0] = up[0] ? j : cls[0];
      v[0] = fmaxf(x, v[0]);
    }
  }
  Stat a{m, 0.f, 0.f};
#pragma unroll 8
  for (int j = 0; j < C; ++j) {
    const float y = fmaxf((z[j] - m) * kL, kFloor), p = ex2(y);
    a.s += p;
    a.t = fmaf(p, y, a.t);
  }
  const int64_t row = r0 + lane;
  const float ls = write_stats<STORE>(o, row, C, Z, C, a, true);
  if constexpr (K > 0) {
    if (cls[K - 1] < 0) {   // fewer than K classes above -Inf: then those at -Inf, ascending
      int f = 0;
#pragma unroll
      for (int k = 0; k < K; ++k) f += cls[k] >= 0;
      for (int j = 0; j < C && f < K; ++j)
        if (z[j] == -INFINITY) {
#pragma unroll
          for (int k = 0; k < K; ++k) cls[k] = k == f ? j : cls[k];
          ++f;
        }
    }
#pragma unroll
    for (int k = 0; k < K; ++k) write_top(o, row, K, k, order_bits(v[k]), static_cast<unsigned>(cls[k]), m, ls);
  }
}

template <int STORE>
void lane_rows(hipStream_t st, int64_t n, int C, const void* Z, const Out& o, int K) {
  const dim3 g(static_cast<unsigned>((n + 63) / 64));
  const unsigned inv = ((1u << 20) + C - 1) / C;
  const unsigned lds = (64 * (C | 1) + 8) * 4;
  switch (K) {
#define LANE(K)                                                  \
  case K:                                                        \
    lane_rows_kernel<STORE, K><<<g, 64, lds, st>>>(n, C, inv, Z, o); \
    break
    LANE(0); LANE(1); LANE(2); LANE(3); LANE(4); LANE(5); LANE(6); LANE(7); LANE(8);
#undef LANE
  }
}

// ---- rows of up to 1,024 classes: LPR lanes a row, E classes a lane ----------------

template <int CTRL>
__device__ __forceinline__ float dpp_f(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(x), __float_as_int(x), CTRL, 0xf, 0xf, false));
}
template <int CTRL>
__device__ __forceinline__ unsigned dpp_u(unsigned x) {
  return static_cast<unsigned>(__builtin_amdgcn_update_dpp(static_cast<int>(x), static_cast<int>(x), CTRL, 0xf, 0xf, false));
}
// f over the LPR lanes of a row, every lane with the result (f commutative).
// Within 16 lanes by lane permutations (swaps in a quad, then mirrors of 8 and
// 16), which cost an instruction each.
template <int LPR, class F>
__device__ __forceinline__ float reduce_f(float x, F f) {
  x = f(x, dpp_f<0xB1>(x));
  x = f(x, dpp_f<0x4E>(x));
  x = f(x, dpp_f<0x141>(x));
  if constexpr (LPR > 8) x = f(x, dpp_f<0x140>(x));
  if constexpr (LPR > 16) x = f(x, __shfl_xor(x, 16, 64));
  if constexpr (LPR > 32) x = f(x, __shfl_xor(x, 32, 64));
  return x;
}
template <int LPR, class F>
__device__ __forceinline__ unsigned reduce_u(unsigned x, F f) {
  x = f(x, dpp_u<0xB1>(x));
  x = f(x, dpp_u<0x4E>(x));
  x = f(x, dpp_u<0x141>(x));
  if constexpr (LPR > 8) x = f(x, dpp_u<0x140>(x));
  if constexpr (LPR > 16) x = f(x, static_cast<unsigned>(__shfl_xor(static_cast<int>(x), 16, 64)));
  if constexpr (LPR > 32) x = f(x, static_cast<unsigned>(__shfl_xor(static_cast<int>(x), 32, 64)));
  return x;
}

// A row is in registers, so its maximum comes first and nothing is rescaled; the
// K best are taken out one by one.  What bounds it: issue (a round of the K best
// is about 5 E + 10 instructions for 64 / LPR rows).  232,965 rows of 47 classes with the
// five best take 21 us.
template <int STORE, int LPR, int E, bool TOP>
__global__ __launch_bounds__(kBlock) void short_rows_kernel(int64_t n, int C, const void* __restrict__ Z,
                                                            int64_t ldz, Out o, int K) {
  constexpr int RPB = kBlock / LPR;
  const int l = threadIdx.x & (LPR - 1);
  // rows of a wave in step: all its lanes reach the permutations below
  for (int64_t r0 = static_cast<int64_t>(blockIdx.x) * RPB; r0 < n; r0 += static_cast<int64_t>(gridDim.x) * RPB) {
    const int64_t row = r0 + threadIdx.x / LPR;
    const bool live = row < n;
    float z[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      float x[1] = {-INFINITY};
      if (live && l + LPR * e < C) load_vec<STORE, 1>(Z, row * ldz + l + LPR * e, x);
      z[e] = x[0];
    }
    Stat a{z[0], 0.f, 0.f};
#pragma unroll
    for (int e = 1; e < E; ++e) a.m = max_nan(a.m, z[e]);
    a.m = reduce_f<LPR>(a.m, [](float x, float y) { return max_nan(x, y); });
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float y = fmaxf((z[e] - a.m) * kL, kFloor), p = ex2(y);
      a.s += p;
      a.t = fmaf(p, y, a.t);
    }
    a.s = reduce_f<LPR>(a.s, [](float x, float y) { return x + y; });
    a.t = reduce_f<LPR>(a.t, [](float x, float y) { return x + y; });
    const float ls = write_stats<STORE>(o, row, C, Z, ldz, a, live && l == 0);
    if constexpr (TOP) {
      unsigned key[E];
#pragma unroll
      for (int e = 0; e < E; ++e) key[e] = l + LPR * e < C ? order_bits(z[e]) : 0u;
      unsigned kb = 0, kc = 0;   // this lane's share of the last LPR results
      for (int k = 0; k < K; ++k) {
        unsigned best = key[0];
#pragma unroll
        for (int e = 1; e < E; ++e) best = max(best, key[e]);
        best = reduce_u<LPR>(best, [](unsigned x, unsigned y) { return max(x, y); });
        unsigned c = 0xffffffffu;
#pragma unroll
        for (int e = E - 1; e >= 0; --e) c = key[e] == best ? static_cast<unsigned>(l + LPR * e) : c;
        c = reduce_u<LPR>(c, [](unsigned x, unsigned y) { return min(x, y); });
#pragma unroll
        for (int e = 0; e < E; ++e) key[e] = static_cast<unsigned>(l + LPR * e) == c ? 0u : key[e];
        if ((k & (LPR - 1)) == l) {
          kb = best;
          kc = c;
        }
        if ((k & (LPR - 1)) == LPR - 1 || k == K - 1) {
          const int at = (k & ~(LPR - 1)) + l;
          if (live && at <= k) write_top(o, row, K, at, kb, kc, a.m, ls);
        }
      }
    }
  }
}

// ---- longer rows ---------------------------------------------------------------------

// One workgroup per (row, part of the row).  parts == 1 writes the outputs,
// else the part's statistics (4 floats) and list (K integers) go to `part`.
// Bound by memory, and for 16-bit logits by issue beside it: 4,093 rows of 50,001
// floats with the eight best 164 us (5.0 TB/s; 316 with 4-byte loads, which an odd
// width took), 8,192 of 32,000 bf16 without any 131 us (4.0 TB/s).  One row of
// 131,072 bf16 with the 20 best, in 32 parts and a join, 14.7 us; 44.6 with lists begun
// by insertions and moved by LDS shuffles.
template <int STORE, bool TOP>
__global__ __launch_bounds__(kBlock) void rows_kernel(int64_t items, int parts, int64_t len, int C,
                                                      const void* __restrict__ Z, int64_t ldz,
                                                      Out o, int K, float* __restrict__ pstat,
                                                      u64* __restrict__ ptop) {
  constexpr int V = STORE == GIST_STORE_F32 ? 4 : 8, kU = 2;
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
    // kU vectors a step: both loads are out before either is used, and the sums
    // are rescaled once for both
    for (int64_t j0 = c0; j0 < c1; j0 += kU * V * kBlock) {   // block-uniform: ballots inside
      float z[kU][V], m = -INFINITY;
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const int64_t j = j0 + (u * kBlock + t) * V;
        load_some<STORE, V>(Z, row * ldz + j, c1 - j, -INFINITY, z[u]);
      }
#pragma unroll
      for (int u = 0; u < kU; ++u)
#pragma unroll
        for (int q = 0; q < V; ++q) m = max_nan(m, z[u][q]);
      if constexpr (TOP) {
        const bool first = j0 == c0;
        int at = -1;
        if (first) {
          // The list begins with the lanes' best: most others then fail its K-th.
          u64 best = 0;
#pragma unroll
          for (int u = 0; u < kU; ++u)
#pragma unroll
            for (int q = 0; q < V; ++q) {
              const int64_t j = j0 + (u * kBlock + t) * V + q;
              const u64 x = j < c1 ? pack(z[u][q], static_cast<unsigned>(j)) : 0;
              if (x > best) {
                best = x;
                at = u * V + q;
              }
            }
          top.sort(best, lane);
        }
        if (__any(pack(m, 0u) > top.thr)) {
#pragma unroll
          for (int u = 0; u < kU; ++u)
#pragma unroll
            for (int q = 0; q < V; ++q) {
              const int64_t j = j0 + (u * kBlock + t) * V + q;
              top.offer(j < c1 && u * V + q != at ? pack(z[u][q], static_cast<unsigned>(j)) : 0, lane);
            }
        }
      }
      rescale(a, max_nan(a.m, m));
#pragma unroll
      for (int u = 0; u < kU; ++u)
#pragma unroll
        for (int q = 0; q < V; ++q) {
          const float y = fmaxf((z[u][q] - a.m) * kL, kFloor);
          const float e = ex2(y);
          a.s += e;
          a.t = fmaf(e, y, a.t);
        }
    }
    a = wave_merge(a);
    __syncthreads();   // the previous item's LDS is read
    if (lane == 0) wst[wave] = a;
    if (TOP) wtop[wave][63 - lane] = lane < K ? top.mine : 0;
    __syncthreads();
    if (wave == 0) {
#pragma unroll
      for (int w = 1; w < kWaves; ++w) {
        merge(a, wst[w]);
        if (TOP) top.join(wtop[w][lane], lane);
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

// Joins the parts of a row: each wave a share of them, then the first wave.  32 parts of the
// 20 best: 6.8 us, 7.8 with one list on its way at a time (lists joined in pairs, fewer one
// after another, made no difference).
template <int STORE>
__global__ __launch_bounds__(kBlock) void join_rows_kernel(int64_t n, int parts, int C,
                                                           const void* __restrict__ Z, int64_t ldz,
                                                           Out o, int K,
                                                           const float* __restrict__ pstat,
                                                           const u64* __restrict__ ptop) {
  constexpr int kU = 8;
  __shared__ u64 wtop[kWaves][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
    Stat a{-INFINITY, 0.f, 0.f};
    for (int p = lane; p < parts; p += 64) {
      const float* s = pstat + 4 * (row * parts + p);
      merge(a, Stat{s[0], s[1], s[2]});
    }
    a = wave_merge(a);
    Top top;
    top.K = K > 0 ? K : 1;
    if (K > 0) {
      for (int p = wave; p < parts; p += kU * kWaves) {   // kU lists on their way at once
        u64 x[kU];
#pragma unroll
        for (int u = 0; u < kU; ++u) {
          const int q = p + u * kWaves;
          x[u] = q < parts && 63 - lane < K ? ptop[(row * parts + q) * K + 63 - lane] : 0;
        }
#pragma unroll
        for (int u = 0; u < kU; ++u)
          if (p + u * kWaves < parts) top.join(x[u], lane);
      }
      __syncthreads();   // the previous row's lists are read
      wtop[wave][63 - lane] = top.mine;
      __syncthreads();
      if (wave == 0)
        for (int w = 1; w < kWaves; ++w) top.join(wtop[w][lane], lane);
    }
    if (wave == 0) write_row<STORE>(o, row, C, Z, ldz, a, top, K, lane);
  }
}

// dz = g_l (1[j = y] - p) - g_H p (log p + H), p = exp(z - lse).  A group of
// 1 << tl threads per (row, slab of columns): 64 lanes of a wave or fewer, or the block.
// An lse beyond kFar has lost bits of log s (2^-19 and more), so the group sums the row's
// exp(z - lse) first, 1 but for that, and takes its logarithm off.  Each group that does so
// reads the whole row, so such a row goes to at most `far` groups, of `far_len` columns
// each, and its other groups have nothing to do: two reads and a write per element.
// Bound by memory: 8,192 x 32,000 bf16 in 183 us (5.7 TB/s).
constexpr float kFar = 64.f;
template <int STORE, int V>
__global__ __launch_bounds__(kBlock) void bwd_kernel(int64_t items, int slabs, int slab, int far, int far_len,
                                                     int turn, int tl, int C,
                                                     const void* Z, int64_t ldz,
                                                     const int* __restrict__ tokens,
                                                     const float* __restrict__ lse,
                                                     const float* __restrict__ ent,
                                                     const float* __restrict__ gl,
                                                     const float* __restrict__ gh, void* dZ,
                                                     int64_t ldd) {
  __shared__ float sums[kWaves];
  const int lane = threadIdx.x & ((1 << tl) - 1);
  for (int64_t item = (static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x) >> tl; item < items;
       item += (static_cast<int64_t>(gridDim.x) * kBlock) >> tl) {
    const int64_t row = slabs == 1 ? item : item / slabs;
    int part = slabs == 1 ? 0 : static_cast<int>(item - row * slabs);
    int64_t c0 = static_cast<int64_t>(part) * slab, c1 = min<int64_t>(C, c0 + slab);
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
    float ls = 0.f;
    if (!none && !bad && fabsf(l) > kFar) {
      // Workgroups go to the 8 XCDs in turn, and to the 4 shader engines of each: the first
      // parts of all rows, 1 << turn of whose multiples meet mod 32, would leave some idle,
      // so they begin one further after each round of them.
      part -= static_cast<int>(row >> (5 - turn)) & ((1 << turn) - 1);
      part += part < 0 ? slabs : 0;
      if (part >= far) continue;   // more than one part: all of the block's threads
      c0 = static_cast<int64_t>(part) * far_len;
      c1 = min<int64_t>(C, c0 + far_len);
      float s = 0.f;
      for (int64_t j = V * lane; j < C; j += V << tl) {
        float z[V];
        load_some<STORE, V>(Z, row * ldz + j, C - j, -INFINITY, z);
#pragma unroll
        for (int q = 0; q < V; ++q) s += ex2(fmaxf(z[q] - l, -200.f) * kL);
      }
      for (int o = min(32, (1 << tl) >> 1); o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
      if (tl == 8) {   // the block's threads have one item
        __syncthreads();   // the last item's sums are read
        if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
        __syncthreads();   // and in place, the row is read
        s = (sums[0] + sums[1]) + (sums[2] + sums[3]);
      }
      ls = kLn2 * lg2(s);
    }
    for (int64_t j = c0 + V * lane; j < c1; j += V << tl) {
      float z[V], d[V];
      load_some<STORE, V>(Z, row * ldz + j, c1 - j, 0.f, z);
#pragma unroll
      for (int q = 0; q < V; ++q) {
        const float x = fmaxf((z[q] - l) - ls, -200.f);
        const float p = ex2(x * kL);
        d[q] = -p * fmaf(w1, x, w0);
        if (none) d[q] = 0.f;
        if (j + q == y) d[q] += gy;
        if (bad) d[q] = __uint_as_float(0x7fc00000u);
      }
      store_some<STORE, V>(dZ, row * ldd + j, c1 - j, d);
    }
  }
}

// Groups that far rows go to together: each reads its whole row, so more of them cost more
// where there are many rows, and fewer leave compute units idle where there are few.  us with
// 256, 512, 1,024 and with every group of every row, fp32: 64 rows of 131,072 classes 70, 65, 67
// and 66, 256 of them 135, 109, 118 and 185, 1,100 of them 400, 405, 404 and 868, 40 of 1,000,003
// 550, 538, 545 and 1,239 (not far: 12, 42, 206 and 55).  Rounded up: 300 rows of 1,000,003 take
// 1,363, 1,577 with one group each.
constexpr int64_t kFarGroups = 512;

struct Plan {
  int parts;
  int64_t len;
};

constexpr int64_t kShort = 1024;   // classes that short_rows_kernel takes

constexpr int64_t kManyRows = 1024;   // rows from which each is one part

int64_t most_parts(int64_t C) { return std::max<int64_t>(1, std::min<int64_t>(C / 4096, 256)); }

// Parts of a row: as many as fill the card, of at least 4,096 elements each
// (16 per thread).
Plan plan_rows(int64_t n, int64_t C) {
  Plan p{1, C};
  if (C <= kShort) return p;
  const int64_t want = n >= kManyRows ? 1 : (kManyRows + n - 1) / std::max<int64_t>(n, 1);
  p.parts = static_cast<int>(std::min(want, most_parts(C)));
  p.len = ((C + p.parts - 1) / p.parts + 7) / 8 * 8;
  p.parts = static_cast<int>((C + p.len - 1) / p.len);
  return p;
}

size_t up256(size_t x) { return (x + 255) & ~size_t(255); }

// Statistics and lists of so many parts.
size_t part_bytes(int64_t parts, int K) {
  return up256(static_cast<size_t>(parts) * 16) + static_cast<size_t>(parts) * K * 8;
}

}  // namespace

size_t log_probs_need(int64_t n, int64_t C, int K) {
  const Plan p = plan_rows(n, C);
  if (p.parts == 1) return 0;
  return part_bytes(n * p.parts, K);
}

// Room for any number of rows up to n: the fewer they are, the more parts a row has.  n rows
// of ceil(1024 / n) parts are fewer than n + 1024.
size_t log_probs_workspace(int64_t n, int64_t C, int K) {
  const int64_t most = most_parts(C);
  if (most == 1) return 0;
  n = std::min(n, kManyRows - 1);
  return part_bytes(std::min(n * most, n + kManyRows - 1), K);
}

gist_status log_probs(hipStream_t st, int64_t n, int64_t C, const void* Z, int64_t ldz, int store,
                      const int32_t* tokens, float* logp, float* entropy, float* lse, int K,
                      float* top_logp, int32_t* top_idx, void* ws) {
  const Plan p = plan_rows(n, C);
  const int eb = store == GIST_STORE_F32 ? 4 : 2, c = static_cast<int>(C);
  const Out o{tokens, logp, entropy, lse, top_logp, top_idx};
  float* pstat = static_cast<float*>(ws);
  u64* ptop = p.parts == 1 ? nullptr
                           : reinterpret_cast<u64*>(static_cast<char*>(ws) +
                                                    up256(static_cast<size_t>(n) * p.parts * 16));
  const int64_t items = n * p.parts;
  ProfScope ps(st, "log_probs", 6.0 * n * C, static_cast<double>(n) * C * eb);
#define BY_STORE(CALL)                                      \
  do {                                                      \
    if (store == GIST_STORE_F32) CALL(GIST_STORE_F32);      \
    else if (store == GIST_STORE_BF16) CALL(GIST_STORE_BF16); \
    else CALL(GIST_STORE_F16);                              \
  } while (0)
  if (n >= kLaneRows && C <= kLaneClasses && K <= kLaneTop && ldz == C) {
#define LANES(S) lane_rows<S>(st, n, c, Z, o, K)
    BY_STORE(LANES);
#undef LANES
    return check_launch("log_probs");
  }
  if (C <= kShort) {
#define SHORT2(S, L, E, T)                                                                         \
  short_rows_kernel<S, L, E, T>                                                                    \
      <<<dim3(static_cast<unsigned>(std::min<int64_t>((n + kBlock / L - 1) / (kBlock / L), 1 << 20))), \
         kBlock, 0, st>>>(n, c, Z, ldz, o, K)
#define SHORT1(S, L, E)                 \
  do {                                  \
    if (K > 0) SHORT2(S, L, E, true);   \
    else SHORT2(S, L, E, false);        \
  } while (0)
#define SHORT(S)                        \
  do {                                  \
    if (C <= 8) SHORT1(S, 8, 1);        \
    else if (C <= 16) SHORT1(S, 8, 2);  \
    else if (C <= 32) SHORT1(S, 8, 4);  \
    else if (C <= 48) SHORT1(S, 8, 6);  \
    else if (C <= 64) SHORT1(S, 8, 8);  \
    else if (C <= 128) SHORT1(S, 16, 8); \
    else if (C <= 256) SHORT1(S, 32, 8); \
    else if (C <= 512) SHORT1(S, 64, 8); \
    else SHORT1(S, 64, 16);             \
  } while (0)
    BY_STORE(SHORT);
#undef SHORT
#undef SHORT1
#undef SHORT2
    return check_launch("log_probs");
  }
  {
    const dim3 g(static_cast<unsigned>(std::min<int64_t>(items, 1 << 22)));
#define ROWS(S)                                                                                             \
  do {                                                                                                      \
    if (K > 0) rows_kernel<S, true><<<g, kBlock, 0, st>>>(items, p.parts, p.len, c, Z, ldz, o, K, pstat, ptop); \
    else rows_kernel<S, false><<<g, kBlock, 0, st>>>(items, p.parts, p.len, c, Z, ldz, o, K, pstat, ptop);      \
  } while (0)
    BY_STORE(ROWS);
#undef ROWS
  }
  if (p.parts > 1) {
    const dim3 gj(static_cast<unsigned>(std::min<int64_t>(n, 1 << 22)));
#define JOIN(S) join_rows_kernel<S><<<gj, kBlock, 0, st>>>(n, p.parts, c, Z, ldz, o, K, pstat, ptop)
    BY_STORE(JOIN);
#undef JOIN
  }
  return check_launch("log_probs");
}

gist_status log_probs_bwd(hipStream_t st, int64_t n, int64_t C, const void* Z, int64_t ldz,
                          int store, const int32_t* tokens, const float* lse,
                          const float* entropy, const float* g_logp, const float* g_entropy,
                          void* dZ, int64_t ldd) {
  const int eb = store == GIST_STORE_F32 ? 4 : 2, most = store == GIST_STORE_F32 ? 4 : 8;
  // short rows: a class per lane, so that a wave's accesses are one run of bytes
  const int v = C <= 64 ? 1 : most;
  int tl = std::min(8, ceil_log2((C + v - 1) / v));
  if (tl == 7) tl = 6;   // a wave or a block
  // slabs of eight steps where a row takes more than one; in place, where a group may
  // read its whole row before it writes, one
  const int64_t step = static_cast<int64_t>(v) << tl;
  const int64_t slab = C <= 8 * step || dZ == Z ? C : 8 * step;
  const int64_t slabs = (C + slab - 1) / slab, items = n * slabs;
  int64_t far = std::min(slabs, (kFarGroups + n - 1) / n);
  const int64_t far_len = std::min(C, ((C + far - 1) / far + step - 1) / step * step);
  far = (C + far_len - 1) / far_len;
  int turn = 0;   // 1 << turn: the largest power of two, up to 32, that divides slabs
  while (turn < 5 && slabs % (int64_t{2} << turn) == 0) ++turn;
  const dim3 g(static_cast<unsigned>(std::min<int64_t>(((items << tl) + kBlock - 1) / kBlock, 1 << 22)));
  ProfScope ps(st, "log_probs_bwd", 8.0 * n * C, 2.0 * n * C * eb);
#define BWD(S, W)                                                                                 \
  bwd_kernel<S, W><<<g, kBlock, 0, st>>>(items, static_cast<int>(slabs), static_cast<int>(slab),      \
                                         static_cast<int>(far), static_cast<int>(far_len), turn, tl,  \
                                         static_cast<int>(C), Z, ldz, tokens, lse, entropy, g_logp,  \
                                         g_entropy, dZ, ldd)
  if (store == GIST_STORE_F32) {
    if (v == 4) BWD(GIST_STORE_F32, 4);
    else BWD(GIST_STORE_F32, 1);
  } else if (store == GIST_STORE_BF16) {
    if (v == 8) BWD(GIST_STORE_BF16, 8);
    else BWD(GIST_STORE_BF16, 1);
  } else {
    if (v == 8) BWD(GIST_STORE_F16, 8);
    else BWD(GIST_STORE_F16, 1);
  }
#undef BWD
#undef BY_STORE
  return check_launch("log_probs_bwd");
}

}  // namespace gist
