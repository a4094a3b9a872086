// Root-mean-square norm with the residual's addition, its gradients, and rows
// in 8 bits.
//
//   h = x + r (rounded to its store),  s = (mean_j h_j^2 + eps)^-1/2,  y = h s g;
//   with u = dy g and n = h s:  dx = s (u - n mean_j(u_j n_j)) + dsum,  dg = sum_v dy n.
//
// All of it is bound by memory: every array is read or written once.  A row is
// held in the registers of 16 lanes, a wave, or a workgroup of 256 or 1,024; longer
// rows are read twice (three times for codes).  Sums are fp32.  Both directions move 4.5 to 5 TB/s where
// rows are whole 16-byte loads: 65,537 rows of 2,048 from fp32 to codes 134 us, 16,384 of 4,096 in bf16 with
// residual and gradients 209 us.  Held by a wave or 256 threads only, 32 elements a thread and a
// branch a load, with long rows read again, these took 183 and 220 us, 100,000 rows of 64 in fp32
// 49 us (now 11), and 4,000 of 16,384 in bf16 180 us (now 111).
//
// 8-bit rows: e4m3, the row's largest magnitude at 448, nearest even.  The codes are those of 64-bit
// arithmetic on h and g, h g (448 / the largest) (s cancels): 32 bits decide all but those near the middle between
// two codes, which are decided again in 64 bits (one element in 60,000 with a norm, in 150,000 without; of
// bf16 rows without one 1 in 200 is a middle itself).  65,537 rows of 2,048 from fp32 take
// 134 us with that and without, 16,384 of 4,096 in bf16 with a residual 114 and 95.
//
// The gain's gradient: a workgroup keeps its rows' sum of dy n in registers (every
// thread has the same columns in each of its rows), writes it once, and a second
// launch adds the workgroups' sums in order: the same bits every time.

#include <algorithm>

#include "elem.cuh"

namespace gist {

namespace {

constexpr int kBlock = 256;
constexpr int kWide = 1024;               // threads of a workgroup whose rows 256 do not hold
constexpr float kTop = 448.f;             // largest e4m3 value
constexpr int64_t kMostBlocks = 1 << 16;  // rows go around them

typedef unsigned u32u __attribute__((aligned(1)));

constexpr int block_of(int threads) { return threads < kBlock ? kBlock : threads; }

template <int STORE>
constexpr int vec_of() { return STORE == GIST_STORE_F32 ? 4 : 8; }

// Sums over the THREADS threads of a row, in a fixed order.  `sh`: two floats a wave, used in
// turn (`turn` flips), so that one barrier a sum is enough.
template <int THREADS>
__device__ __forceinline__ float row_sum(float v, float* sh, int& turn) {
  if constexpr (THREADS < 64) {
#pragma unroll
    for (int o = THREADS / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
  }
  v = wave_sum(v);
  if constexpr (THREADS == 64) return v;
  float* s = sh + turn * (THREADS / 64);
  turn ^= 1;
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.f;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) v += s[w];
  return v;
}
// The largest of magnitudes; as integers their bits are in the same order, and a NaN's are
// above all others'.
template <int THREADS>
__device__ __forceinline__ float row_max(float m, float* sh, int& turn) {
  int v = __float_as_int(m);
#pragma unroll
  for (int o = (THREADS < 64 ? THREADS : 64) / 2; o > 0; o >>= 1) v = max(v, __shfl_xor(v, o, 64));
  if constexpr (THREADS <= 64) return __int_as_float(v);
  float* s = sh + turn * (THREADS / 64);
  turn ^= 1;
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = __int_as_float(v);
  __syncthreads();
  v = __float_as_int(s[0]);
#pragma unroll
  for (int w = 1; w < THREADS / 64; ++w) v = max(v, __float_as_int(s[w]));
  return __int_as_float(v);
}
__device__ __forceinline__ float larger(float big, float y) {
  return __int_as_float(max(__float_as_int(big), __float_as_int(fabsf(y))));
}

// V values times inv as e4m3 codes, the first `left` of them stored.
template <int V>
__device__ __forceinline__ void store_e4m3(void* base, int64_t e, int64_t left, const float (&y)[V], float inv) {
  unsigned char* p = static_cast<unsigned char*>(base) + e;
#pragma unroll
  for (int h = 0; h < V; h += 4) {
    // |y inv| <= 448 (1 + 2^-23), which rounds to 448 (as all up to 464 do); NaN stays
    int u = __builtin_amdgcn_cvt_pk_fp8_f32(y[h] * inv, y[h + 1] * inv, 0, false);
    u = __builtin_amdgcn_cvt_pk_fp8_f32(y[h + 2] * inv, y[h + 3] * inv, u, true);
    if (left >= h + 4) {
      *reinterpret_cast<u32u*>(p + h) = static_cast<unsigned>(u);
    } else {
#pragma unroll
      for (int q = 0; q < 3; ++q)
        if (h + q < left) p[h + q] = static_cast<unsigned char>(u >> (8 * q));
    }
  }
}

struct Fwd {
  int64_t n, ldx, ldr, ldh, ldy;
  int d;
  const void* x;
  const void* r;
  const float* gain;
  void* h;
  void* y;
  float* y_scale;
  float* rstd;
  float eps;
};

template <int STORE, int V>
__device__ __forceinline__ void load_h(const Fwd& a, int64_t row, int c, int left, float (&h)[V]) {
  load_some<STORE, V>(a.x, row * a.ldx + c, left, 0.f, h);
  if (a.r) {
    float r[V];
    load_some<STORE, V>(a.r, row * a.ldr + c, left, 0.f, r);
#pragma unroll
    for (int q = 0; q < V; ++q) {
      h[q] += r[q];
      if constexpr (STORE != GIST_STORE_F32) h[q] = widen<STORE>(narrow<STORE>(h[q]));
    }
  }
}

template <int OUT, int V>
__device__ __forceinline__ void store_y(void* base, int64_t e, int left, const float (&y)[V], float inv) {
  if constexpr (OUT == GIST_STORE_E4M3) {
    store_e4m3<V>(base, e, left, y, inv);
  } else if constexpr (OUT != GIST_STORE_F32 && V == 4) {
    typedef unsigned short us4 __attribute__((ext_vector_type(4), aligned(2)));
    unsigned short* p = static_cast<unsigned short*>(base) + e;
    us4 t;
#pragma unroll
    for (int q = 0; q < 4; ++q) t[q] = narrow<OUT>(y[q]);
    if (left >= 4) {
      *reinterpret_cast<us4*>(p) = t;
    } else {
#pragma unroll
      for (int q = 0; q < 3; ++q)
        if (q < left) p[q] = t[q];
    }
  } else {
    store_some<OUT, V>(base, e, left, y);
  }
}

// A row's scale from its largest magnitude, and what takes its values to codes.  A row that
// holds a NaN or an Inf is NaN throughout; one below kLeast is zero.
constexpr float kLeast = 0x1p-100f;
__device__ __forceinline__ float scale_of(float big, float& inv) {
  if (!(big < __builtin_inff())) big = __builtin_nanf("");
  const bool zero = big < kLeast;
  inv = zero ? 0.f : kTop / big;
  return zero ? 0.f : big / kTop;
}

// How far a code's argument is from the middle between two codes, whose 20 lowest bits are
// 0x80000, in units of its last place, times 2^12: at most 2 kNear if within kNear of it.  32 bits leave
// an argument off by less: the quotient's and the product's roundings and, with a norm, two each of it and
// of the row's largest, 2 or 6 of 2^-24 relative, as many places at most.
template <bool NORM>
constexpr unsigned kNear = (NORM ? 8u : 3u) << 12;
template <bool NORM>
__device__ __forceinline__ unsigned border(float a) { return (__float_as_uint(a) << 12) + (0x80000000u + kNear<NORM>); }
// Below 2^-6 codes are 2^-9 apart throughout: 32 |a| + 1/2 has their middles where border looks for them
// (the error is half the places above, and half of one by the addition).  What is larger becomes 1,
// which is no middle.
template <bool NORM>
__device__ __forceinline__ unsigned border_small(float a) {
  return border<NORM>(__builtin_amdgcn_fmed3f(fmaf(fabsf(a), 32.f, 0.5f), 0.f, 1.f));
}

// A float whose nearest code is a's: a cut to 24 bits, the last of them set where something was cut off, so
// that nothing but a middle itself becomes one.
__device__ __forceinline__ float decided(double a) {
  const float f = static_cast<float>(a);
  const double w = static_cast<double>(f);
  if (w == a) return f;
  return __uint_as_float((__float_as_uint(f) - (fabs(w) > fabs(a) ? 1u : 0u)) | 1u);
}

template <int THREADS>
__device__ __forceinline__ double row_max64(double v, double* sh) {
#pragma unroll
  for (int o = (THREADS < 64 ? THREADS : 64) / 2; o > 0; o >>= 1) v = fmax(v, __shfl_xor(v, o, 64));
  if constexpr (THREADS <= 64) return v;
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  v = sh[0];
#pragma unroll
  for (int w = 1; w < THREADS / 64; ++w) v = fmax(v, sh[w]);
  return v;
}

// h times the gain in 64 bits: h from where it has just been stored, since x or the residual may be there.
template <int STORE, bool NORM>
__device__ __forceinline__ double exact_y(const Fwd& a, int64_t row, int c) {
  float h[1];
  if (NORM && a.h) load_vec<STORE, 1>(a.h, row * a.ldh + c, h);
  else load_h<STORE, 1>(a, row, c, 1, h);
  return static_cast<double>(h[0]) * (NORM ? a.gain[c] : 1.f);
}

// Waves of a SIMD at least.  For codes the compiler would take registers for the rare second decision that
// cost the rest its waves: with a residual in bf16 65,537 rows of 2,048 take 181 us with five,
// 198 with four and 245 with six; 100,000 of 602 176 with four, 203 as it pleases; from fp32 65,537 of
// 2,048 134 with four, 206 with five.
constexpr int rows_waves(int store, int out, int threads, bool tail) {
  return out != GIST_STORE_E4M3 ? 1 : threads > kBlock || store == GIST_STORE_F32 || tail ? 4 : 5;
}

// A row in the registers of THREADS threads: CH loads of V elements each and, with TAIL, one element each
// of what those leave (a load that may end inside a row takes a branch a load: 183 us for
// 65,537 rows of 2,048 from fp32 to codes, 134 without; of 602, with a residual, 147 and 116).  NORM false: no norm, the row's codes alone.
template <int STORE, int OUT, int THREADS, int CH, bool NORM, bool TAIL>
__global__ __launch_bounds__(block_of(THREADS), rows_waves(STORE, OUT, THREADS, TAIL)) void rows_kernel(Fwd a) {
  constexpr int V = vec_of<STORE>();
  __shared__ float sh[2 * block_of(THREADS) / 64];
  __shared__ double sh64[OUT == GIST_STORE_E4M3 ? block_of(THREADS) / 64 : 1];
  int turn = 0;
  const int lane = threadIdx.x % THREADS;
  const int whole = TAIL ? a.d - a.d % V : a.d, tail = whole + lane;
  const float inv_d = 1.f / static_cast<float>(a.d);
  constexpr int RB = block_of(THREADS) / THREADS;
  for (int64_t row = blockIdx.x * RB + threadIdx.x / THREADS; row < a.n; row += static_cast<int64_t>(gridDim.x) * RB) {
    float h[CH][V], t[1] = {0.f};
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = (i * THREADS + lane) * V;
#pragma unroll
      for (int q = 0; q < V; ++q) h[i][q] = 0.f;
      if (c < whole) load_h<STORE, V>(a, row, c, V, h[i]);
    }
    if (TAIL && tail < a.d) load_h<STORE, 1>(a, row, tail, 1, t);
    float big = 0.f;
    if constexpr (NORM) {
      float s = TAIL ? t[0] * t[0] : 0.f;
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        float p = 0.f;
#pragma unroll
        for (int q = 0; q < V; ++q) p = fmaf(h[i][q], h[i][q], p);
        s += p;
      }
      const float rstd = 1.f / sqrtf(row_sum<THREADS>(s, sh, turn) * inv_d + a.eps);
      if (a.rstd && lane == 0) a.rstd[row] = rstd;
      int at = lane;
      // the gain's addresses, kept over the rows, would have registers of the codes spilled
      if constexpr (OUT == GIST_STORE_E4M3 && STORE != GIST_STORE_F32) asm volatile("" : "+v"(at));
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const int c = (i * THREADS + at) * V;
        if (c >= whole) continue;
        if (a.h) store_as<STORE, V>(a.h, row * a.ldh + c, h[i]);
        float g[V];
#pragma unroll
        for (int q = 0; q < V; q += 4) {
          float u[4];
          load_vec<GIST_STORE_F32, 4>(a.gain, c + q, u);
#pragma unroll
          for (int k = 0; k < 4; ++k) g[q + k] = u[k];
        }
#pragma unroll
        for (int q = 0; q < V; ++q) h[i][q] = h[i][q] * rstd * g[q];
        if constexpr (OUT != GIST_STORE_E4M3) store_y<OUT, V>(a.y, row * a.ldy + c, V, h[i], 0.f);
      }
      if (TAIL && tail < a.d) {
        if (a.h) store_as<STORE, 1>(a.h, row * a.ldh + tail, t);
        t[0] = t[0] * rstd * a.gain[tail];
        if constexpr (OUT != GIST_STORE_E4M3) store_as<OUT, 1>(a.y, row * a.ldy + tail, t);
      }
    }
    if constexpr (OUT == GIST_STORE_E4M3) {
      if (TAIL) big = larger(big, t[0]);
#pragma unroll
      for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int q = 0; q < V; ++q) big = larger(big, h[i][q]);
      float inv;
      const float scale = scale_of(row_max<THREADS>(big, sh, turn), inv);
      if (lane == 0) a.y_scale[row] = scale;
      unsigned near = ~0u, near_small = ~0u;
#pragma unroll
      for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int q = 0; q < V; ++q) {
          h[i][q] *= inv;
          near = min(near, border<NORM>(h[i][q]));
          near_small = min(near_small, border_small<NORM>(h[i][q]));
        }
      if (TAIL) {
        t[0] *= inv;
        near = min(near, border<NORM>(t[0]));
        near_small = min(near_small, border_small<NORM>(t[0]));
      }
      bool again;
      if constexpr (THREADS <= 64) again = __any(min(near, near_small) <= 2 * kNear<NORM>);
      else again = __syncthreads_or(min(near, near_small) <= 2 * kNear<NORM>);
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const int c = (i * THREADS + lane) * V;
        if (c < whole) store_y<OUT, V>(a.y, row * a.ldy + c, V, h[i], 1.f);
      }
      if (TAIL && tail < a.d)
        static_cast<unsigned char*>(a.y)[row * a.ldy + tail] =
            static_cast<unsigned char>(__builtin_amdgcn_cvt_pk_fp8_f32(t[0], 0.f, 0, false));
      if (again) {
        // the largest is one of those that 32 bits put next to it; then what is near a middle, over
        // the codes that have been stored; where a thread has a small one near a middle, all of its own (a second
        // test of every element here took 12 us of 94, 65,537 rows of 2,048 in bf16)
        constexpr float kLargest = kTop * (1.f - 0x1p-20f);
        static_assert(CH * V <= 32, "a bit for each of a thread's elements");
        unsigned large = 0u, close = 0u;
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
          for (int q = 0; q < V; ++q) {
            float x = h[i][q];
            asm volatile("" : "+v"(x));   // from h again: no value of the tests above is kept for this
            if (fabsf(x) > kLargest) large |= 1u << (i * V + q);
            if (border<NORM>(x) <= 2 * kNear<NORM>) close |= 1u << (i * V + q);
          }
        const bool all = near_small <= 2 * kNear<NORM>;
        if (all) close = ~0u >> (32 - CH * V);
        auto column = [&](int e) { return (e / V * THREADS + lane) * V + e % V; };
        double big64 = 0.0;
#pragma unroll 1
        for (; large; large &= large - 1u)
          big64 = fmax(big64, fabs(exact_y<STORE, NORM>(a, row, column(__ffs(large) - 1))));
        if (TAIL && fabsf(t[0]) > kLargest) big64 = fmax(big64, fabs(exact_y<STORE, NORM>(a, row, tail)));
        const double inv64 = 448.0 / row_max64<THREADS>(big64, sh64);
        auto again_at = [&](int c) {
          static_cast<unsigned char*>(a.y)[row * a.ldy + c] = static_cast<unsigned char>(
              __builtin_amdgcn_cvt_pk_fp8_f32(decided(exact_y<STORE, NORM>(a, row, c) * inv64), 0.f, 0, false));
        };
        if (inv > 0.f) {     // no row of zeros or NaN
#pragma unroll 1
          for (; close; close &= close - 1u) {
            const int c = column(__ffs(close) - 1);
            if (c < whole) again_at(c);
          }
          if (TAIL && tail < a.d && (all || border<NORM>(t[0]) <= 2 * kNear<NORM>)) again_at(tail);
        }
      }
    }
  }
}

// Rows longer than a workgroup's registers: read again from x and r for each pass; all
// codes in 64 bits.
template <int STORE, int OUT, bool NORM>
__global__ __launch_bounds__(kBlock) void long_rows_kernel(Fwd a) {
  constexpr int V = vec_of<STORE>();
  __shared__ float sh[2 * kBlock / 64];
  __shared__ double sh64[OUT == GIST_STORE_E4M3 ? kBlock / 64 : 1];
  int turn = 0;
  const float inv_d = 1.f / static_cast<float>(a.d);
  for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
    float rstd = 1.f;
    if constexpr (NORM) {
      float s = 0.f;
      for (int64_t c = threadIdx.x * V; c < a.d; c += kBlock * V) {
        float h[V], p = 0.f;
        load_h<STORE, V>(a, row, c, a.d - c, h);
#pragma unroll
        for (int q = 0; q < V; ++q) p = fmaf(h[q], h[q], p);
        s += p;
      }
      rstd = 1.f / sqrtf(row_sum<kBlock>(s, sh, turn) * inv_d + a.eps);
      if (a.rstd && threadIdx.x == 0) a.rstd[row] = rstd;
    }
    float big = 0.f, inv = 0.f;
    double big64 = 0.0, inv64 = 0.0;
    // for codes: first the largest magnitude, then the codes
    for (int pass = OUT == GIST_STORE_E4M3 ? 0 : 1; pass < 2; ++pass) {
      for (int64_t c = threadIdx.x * V; c < a.d; c += kBlock * V) {
        float h[V];
        const int left = static_cast<int>(min(static_cast<int64_t>(V), a.d - c));
        load_h<STORE, V>(a, row, c, left, h);
        float y[V], g[V];
#pragma unroll
        for (int q = 0; q < V; ++q) {
          g[q] = q >= left ? 0.f : NORM ? a.gain[c + q] : 1.f;
          y[q] = NORM ? h[q] * rstd * g[q] : h[q];
        }
        if (pass == 0) {
#pragma unroll
          for (int q = 0; q < V; ++q) {
            big = larger(big, y[q]);
            big64 = fmax(big64, fabs(static_cast<double>(h[q]) * g[q]));
          }
        } else {
          if constexpr (OUT == GIST_STORE_E4M3) {
#pragma unroll
            for (int q = 0; q < V; ++q)
              y[q] = inv > 0.f ? decided(static_cast<double>(h[q]) * g[q] * inv64) : copysignf(inv, h[q]);
          }
          store_y<OUT, V>(a.y, row * a.ldy + c, left, y, 1.f);
          if (NORM && a.h) store_some<STORE, V>(a.h, row * a.ldh + c, left, h);
        }
      }
      if (pass == 0) {
        const float scale = scale_of(row_max<kBlock>(big, sh, turn), inv);
        if (threadIdx.x == 0) a.y_scale[row] = scale;
        inv64 = 448.0 / row_max64<kBlock>(big64, sh64);
      }
    }
  }
}

struct Bwd {
  int64_t n, lddy, ldh, ldds, lddx;
  int d;
  const void* dy;
  const void* h;
  const float* gain;
  const float* rstd;
  const void* dsum;
  void* dx;
  float* part;      // [grid][d]
  const int32_t* labels;   // or NULL
  const int32_t* n_dev;    // or NULL
};

// Whether a row takes part.  Where it does not, h, dy and rstd become zeros by selection before anything
// is computed with them: 0 times a NaN would be a NaN in every row's gain.
__device__ __forceinline__ int64_t rows_real(const Bwd& a) { return a.n_dev ? *a.n_dev : a.n; }
__device__ __forceinline__ bool takes_part(const Bwd& a, int64_t row, int64_t real) {
  return row < real && (!a.labels || a.labels[row] >= 0);
}

// V elements of any store (V as the rows' own loads have it).
template <int STORE, int V>
__device__ __forceinline__ void load_any(const void* base, int64_t e, int left, float (&x)[V]) {
  if constexpr (STORE == GIST_STORE_F32 && V == 8) {
#pragma unroll
    for (int h = 0; h < 8; h += 4) {
      float t[4];
      load_some<STORE, 4>(base, e + h, left - h, 0.f, t);
#pragma unroll
      for (int q = 0; q < 4; ++q) x[h + q] = t[q];
    }
  } else if constexpr (STORE != GIST_STORE_F32 && V == 4) {
    typedef unsigned short us4 __attribute__((ext_vector_type(4), aligned(2)));
    const unsigned short* p = static_cast<const unsigned short*>(base) + e;
    if (left >= 4) {
      const us4 t = *reinterpret_cast<const us4*>(p);
#pragma unroll
      for (int q = 0; q < 4; ++q) x[q] = widen<STORE>(t[q]);
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) x[q] = q < left ? widen<STORE>(p[q]) : 0.f;
    }
  } else {
    load_some<STORE, V>(base, e, left, 0.f, x);
  }
}

template <int STORE, int DY, int THREADS, int CH, bool TAIL>
__global__ __launch_bounds__(block_of(THREADS)) void bwd_kernel(Bwd a) {
  constexpr int V = vec_of<STORE>();
  __shared__ float sh[2 * block_of(THREADS) / 64];
  __shared__ __attribute__((aligned(16))) float join[THREADS <= 64 ? THREADS * (CH * V + 1) : 4];
  int turn = 0;
  const int lane = threadIdx.x % THREADS, sub = threadIdx.x / THREADS;
  const int whole = TAIL ? a.d - a.d % V : a.d, tail = whole + lane;   // as in rows_kernel
  const float inv_d = 1.f / static_cast<float>(a.d);
  constexpr int RB = block_of(THREADS) / THREADS;
  float acc[CH][V] = {}, g[CH][V], acct = 0.f;
  const float gt = TAIL && tail < a.d ? a.gain[tail] : 0.f;
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int c = (i * THREADS + lane) * V;
#pragma unroll
    for (int q = 0; q < V; ++q) g[i][q] = 0.f;
    if (c < whole) load_any<GIST_STORE_F32, V>(a.gain, c, V, g[i]);
  }
  const int64_t real = rows_real(a);
  for (int64_t row = blockIdx.x * RB + sub; row < a.n; row += static_cast<int64_t>(gridDim.x) * RB) {
    const bool part = takes_part(a, row, real);
    const float s = part ? a.rstd[row] : 0.f;
    float h[CH][V], y[CH][V], ht[1] = {0.f}, yt[1] = {0.f};
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = (i * THREADS + lane) * V;
#pragma unroll
      for (int q = 0; q < V; ++q) h[i][q] = y[i][q] = 0.f;
      if (c < whole) {
        load_vec<STORE, V>(a.h, row * a.ldh + c, h[i]);
        load_any<DY, V>(a.dy, row * a.lddy + c, V, y[i]);
      }
    }
    if (TAIL && tail < a.d) {
      load_vec<STORE, 1>(a.h, row * a.ldh + tail, ht);
      load_vec<DY, 1>(a.dy, row * a.lddy + tail, yt);
    }
    if (!part) {
      ht[0] = yt[0] = 0.f;
#pragma unroll
      for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int q = 0; q < V; ++q) h[i][q] = y[i][q] = 0.f;
    }
    float dot = 0.f;
    if constexpr (TAIL) {
      ht[0] *= s;
      acct = fmaf(yt[0], ht[0], acct);
      yt[0] *= gt;
      dot = yt[0] * ht[0];
    }
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int q = 0; q < V; ++q) {
        h[i][q] *= s;
        acc[i][q] = fmaf(y[i][q], h[i][q], acc[i][q]);
        y[i][q] *= g[i][q];
        dot = fmaf(y[i][q], h[i][q], dot);
      }
    dot = row_sum<THREADS>(dot, sh, turn) * inv_d;
    if (a.dx) {
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const int c = (i * THREADS + lane) * V;
        if (c >= whole) continue;
        float z[V];
#pragma unroll
        for (int q = 0; q < V; ++q) z[q] = 0.f;
        if (a.dsum) load_vec<STORE, V>(a.dsum, row * a.ldds + c, z);
#pragma unroll
        for (int q = 0; q < V; ++q) z[q] = fmaf(s, y[i][q] - h[i][q] * dot, z[q]);
        store_as<STORE, V>(a.dx, row * a.lddx + c, z);
      }
      if (TAIL && tail < a.d) {
        float z[1] = {0.f};
        if (a.dsum) load_vec<STORE, 1>(a.dsum, row * a.ldds + tail, z);
        z[0] = fmaf(s, yt[0] - ht[0] * dot, z[0]);
        store_as<STORE, 1>(a.dx, row * a.lddx + tail, z);
      }
    }
  }
  if (!a.part) return;
  if constexpr (THREADS <= 64) {     // the workgroup's rows, in order
    for (int w = 0; w < RB; ++w) {
      if (sub == w) {
        auto add = [&](float& x, float* p) {
          x += w == 0 ? 0.f : *p;
          if (w + 1 < RB) *p = x;
        };
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
          for (int q = 0; q < V; ++q) add(acc[i][q], join + (i * THREADS + lane) * V + q);
        if (TAIL) add(acct, join + THREADS * CH * V + lane);
      }
      if (w + 1 < RB) __syncthreads();
    }
    if (sub != RB - 1) return;
  }
  float* const out = a.part + static_cast<int64_t>(blockIdx.x) * a.d;
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int c = (i * THREADS + lane) * V;
    if (c >= whole) continue;
#pragma unroll
    for (int q = 0; q < V; ++q) out[c + q] = acc[i][q];
  }
  if (TAIL && tail < a.d) out[tail] = acct;
}

// Rows longer than a workgroup's registers: two passes a row; the gain's sums lie in `part`,
// where the same thread adds to the same columns.
template <int STORE, int DY>
__global__ __launch_bounds__(kBlock) void long_bwd_kernel(Bwd a) {
  constexpr int V = vec_of<STORE>();
  __shared__ float sh[2 * kBlock / 64];
  int turn = 0;
  const float inv_d = 1.f / static_cast<float>(a.d);
  float* const out = a.part ? a.part + static_cast<int64_t>(blockIdx.x) * a.d : nullptr;
  bool first = true;
  const int64_t real = rows_real(a);
  for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
    const bool part = takes_part(a, row, real);
    const float s = part ? a.rstd[row] : 0.f;
    float dot = 0.f;
    for (int64_t c = threadIdx.x * V; c < a.d; c += kBlock * V) {
      const int left = static_cast<int>(min(static_cast<int64_t>(V), a.d - c));
      float h[V], y[V];
      load_some<STORE, V>(a.h, row * a.ldh + c, left, 0.f, h);
      load_any<DY, V>(a.dy, row * a.lddy + c, left, y);
#pragma unroll
      for (int q = 0; q < V; ++q) {
        if (q >= left) break;
        h[q] = part ? h[q] * s : 0.f;
        if (!part) y[q] = 0.f;
        const float p = y[q] * h[q];
        if (out) out[c + q] = first ? p : out[c + q] + p;
        dot = fmaf(y[q] * a.gain[c + q], h[q], dot);
      }
    }
    dot = row_sum<kBlock>(dot, sh, turn) * inv_d;
    first = false;
    if (!a.dx) continue;
    for (int64_t c = threadIdx.x * V; c < a.d; c += kBlock * V) {
      const int left = static_cast<int>(min(static_cast<int64_t>(V), a.d - c));
      float h[V], y[V], z[V];
#pragma unroll
      for (int q = 0; q < V; ++q) z[q] = 0.f;
      load_some<STORE, V>(a.h, row * a.ldh + c, left, 0.f, h);
      load_any<DY, V>(a.dy, row * a.lddy + c, left, y);
      if (a.dsum) load_some<STORE, V>(a.dsum, row * a.ldds + c, left, 0.f, z);
#pragma unroll
      for (int q = 0; q < V; ++q) {
        const float g = q < left ? a.gain[c + q] : 0.f;
        if (part) z[q] = fmaf(s, y[q] * g - h[q] * s * dot, z[q]);
      }
      store_some<STORE, V>(a.dx, row * a.lddx + c, left, z);
    }
  }
}

// dgain[c] = sum of `parts` rows of part: 64 columns a workgroup, its 16 groups of 64 threads
// each every 16th row, joined in order.
constexpr int kJoinWaves = 16;
__global__ __launch_bounds__(64 * kJoinWaves) void gain_kernel(int parts, int d, const float* __restrict__ part,
                                                               float* __restrict__ dgain) {
  __shared__ float sh[kJoinWaves][64];
  const int c = blockIdx.x * 64 + (threadIdx.x & 63), w = threadIdx.x >> 6;
  float s = 0.f;
  if (c < d) {
    int p = w;
    for (; p + 3 * kJoinWaves < parts; p += 4 * kJoinWaves) {
      float v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = part[static_cast<int64_t>(p + i * kJoinWaves) * d + c];
      s += (v[0] + v[1]) + (v[2] + v[3]);
    }
    for (; p < parts; p += kJoinWaves) s += part[static_cast<int64_t>(p) * d + c];
  }
  sh[w][threadIdx.x & 63] = s;
  __syncthreads();
  if (w == 0 && c < d) {
    s = 0.f;
#pragma unroll
    for (int i = 0; i < kJoinWaves; ++i) s += sh[i][threadIdx.x];
    dgain[c] = s;
  }
}

constexpr int kFwdCh(int v) { return 32 / v; }   // 32 elements a thread, 16 in the backward pass
constexpr int kBwdCh(int v) { return 16 / v; }

template <int STORE, int OUT, bool NORM, bool TAIL>
void launch_rows_of(hipStream_t st, const Fwd& a) {
  constexpr int CH = kFwdCh(vec_of<STORE>()), few = 8 / vec_of<STORE>();
  // A wave a row leaves more rows in flight (65,537 rows of 2,048 in fp32, to codes: 181 us, 254 by 256
  // threads); 256 threads a row end a few long rows sooner.  Rows of a few hundred elements take eight a
  // thread, not 32 (200,000 rows of 256 in bf16: 63 and 76 us), and 16 lanes where those hold them
  // (300,000 of 41: 26 and 143 us).
  if (a.d <= 16 * 8) {
    const int64_t g = std::min<int64_t>((a.n + 15) / 16, kMostBlocks);
    hipLaunchKernelGGL((rows_kernel<STORE, OUT, 16, few, NORM, TAIL>), dim3(static_cast<unsigned>(g)), dim3(kBlock), 0, st, a);
  } else if (a.d <= 64 * 8) {
    const int64_t g = std::min<int64_t>((a.n + 3) / 4, kMostBlocks);
    hipLaunchKernelGGL((rows_kernel<STORE, OUT, 64, few, NORM, TAIL>), dim3(static_cast<unsigned>(g)), dim3(kBlock), 0, st, a);
  } else if (a.d <= 64 * 32 && a.n >= 1024) {
    const int64_t g = std::min<int64_t>((a.n + 3) / 4, kMostBlocks);
    hipLaunchKernelGGL((rows_kernel<STORE, OUT, 64, CH, NORM, TAIL>), dim3(static_cast<unsigned>(g)), dim3(kBlock), 0, st, a);
  } else if (a.d <= kBlock * 32) {
    const int64_t g = std::min<int64_t>(a.n, kMostBlocks);
    hipLaunchKernelGGL((rows_kernel<STORE, OUT, kBlock, CH, NORM, TAIL>), dim3(static_cast<unsigned>(g)), dim3(kBlock), 0, st, a);
  } else if (a.d <= kWide * 32) {
    const int64_t g = std::min<int64_t>(a.n, kMostBlocks);
    hipLaunchKernelGGL((rows_kernel<STORE, OUT, kWide, CH, NORM, TAIL>), dim3(static_cast<unsigned>(g)), dim3(kWide), 0, st, a);
  } else {
    const int64_t g = std::min<int64_t>(a.n, kMostBlocks);
    hipLaunchKernelGGL((long_rows_kernel<STORE, OUT, NORM>), dim3(static_cast<unsigned>(g)), dim3(kBlock), 0, st, a);
  }
}

template <int STORE, int OUT, bool NORM>
void launch_rows(hipStream_t st, const Fwd& a) {
  if (a.d % vec_of<STORE>() == 0) launch_rows_of<STORE, OUT, NORM, false>(st, a);
  else launch_rows_of<STORE, OUT, NORM, true>(st, a);
}

template <int STORE>
void launch_norm(hipStream_t st, const Fwd& a, int out) {
  if (out == GIST_STORE_F32) launch_rows<STORE, GIST_STORE_F32, true>(st, a);
  else if (out == GIST_STORE_BF16) launch_rows<STORE, GIST_STORE_BF16, true>(st, a);
  else if (out == GIST_STORE_F16) launch_rows<STORE, GIST_STORE_F16, true>(st, a);
  else launch_rows<STORE, GIST_STORE_E4M3, true>(st, a);
}

// Rows a workgroup of the backward pass takes at a time, and workgroups: enough to fill the
// card twice over, no more than rows (their sums are added by a second launch).  Both passes of 16,384 rows of
// 4,096 in bf16: 212 us, 265 by 512 workgroups.
int rows_a_block(int d) { return d <= 16 * 8 ? kBlock / 16 : d <= 64 * 16 ? kBlock / 64 : 1; }
int64_t bwd_blocks(int64_t n, int d) {
  const int64_t rb = rows_a_block(d);
  return std::min<int64_t>((n + rb - 1) / rb, 1024);
}

template <int STORE, int DY, bool TAIL>
void launch_bwd_rows(hipStream_t st, const Bwd& a) {
  constexpr int V = vec_of<STORE>(), CH = kBwdCh(V), few = 8 / V;
  const dim3 grid(static_cast<unsigned>(bwd_blocks(a.n, a.d))), block(kBlock);
  // threads and elements a row as in the forward pass, half as many elements
  if (a.d <= 16 * 8) hipLaunchKernelGGL((bwd_kernel<STORE, DY, 16, few, TAIL>), grid, block, 0, st, a);
  else if (a.d <= 64 * 8) hipLaunchKernelGGL((bwd_kernel<STORE, DY, 64, few, TAIL>), grid, block, 0, st, a);
  else if (a.d <= 64 * 16) hipLaunchKernelGGL((bwd_kernel<STORE, DY, 64, CH, TAIL>), grid, block, 0, st, a);
  else if (a.d <= kBlock * 16) hipLaunchKernelGGL((bwd_kernel<STORE, DY, kBlock, CH, TAIL>), grid, block, 0, st, a);
  else if (a.d <= kWide * 16) hipLaunchKernelGGL((bwd_kernel<STORE, DY, kWide, CH, TAIL>), grid, dim3(kWide), 0, st, a);
  else hipLaunchKernelGGL((long_bwd_kernel<STORE, DY>), grid, block, 0, st, a);
}

template <int STORE, int DY>
void launch_bwd(hipStream_t st, const Bwd& a) {
  if (a.d % vec_of<STORE>() == 0) launch_bwd_rows<STORE, DY, false>(st, a);
  else launch_bwd_rows<STORE, DY, true>(st, a);
}

template <int STORE>
void launch_bwd_of(hipStream_t st, const Bwd& a, int dy_store) {
  if (dy_store == GIST_STORE_F32) launch_bwd<STORE, GIST_STORE_F32>(st, a);
  else if (dy_store == GIST_STORE_BF16) launch_bwd<STORE, GIST_STORE_BF16>(st, a);
  else launch_bwd<STORE, GIST_STORE_F16>(st, a);
}

double width_of(int store) { return store == GIST_STORE_F32 ? 4.0 : store == GIST_STORE_E4M3 ? 1.0 : 2.0; }

}  // namespace

gist_status rms_norm(hipStream_t st, int64_t n, int d, const void* x, int64_t ldx, const void* r, int64_t ldr,
                     int store, const float* gain, float eps, void* h, int64_t ldh, void* y, int64_t ldy,
                     int out_store, float* y_scale, float* rstd) {
  const Fwd a{n, ldx, ldr, ldh, ldy, d, x, r, gain, h, y, y_scale, rstd, eps};
  ProfScope ps(st, "rms_norm", 0.0,
               static_cast<double>(n) * d * (width_of(store) * (1.0 + (r ? 1 : 0) + (h ? 1 : 0)) + width_of(out_store)));
  if (store == GIST_STORE_F32) launch_norm<GIST_STORE_F32>(st, a, out_store);
  else if (store == GIST_STORE_BF16) launch_norm<GIST_STORE_BF16>(st, a, out_store);
  else launch_norm<GIST_STORE_F16>(st, a, out_store);
  return check_launch("rms_norm");
}

gist_status quantize_rows(hipStream_t st, int64_t n, int d, const void* x, int64_t ldx, int store, void* y,
                          int64_t ldy, float* scale) {
  const Fwd a{n, ldx, 0, 0, ldy, d, x, nullptr, nullptr, nullptr, y, scale, nullptr, 0.f};
  ProfScope ps(st, "quantize_rows", 0.0, static_cast<double>(n) * d * (width_of(store) + 1.0));
  if (store == GIST_STORE_F32) launch_rows<GIST_STORE_F32, GIST_STORE_E4M3, false>(st, a);
  else if (store == GIST_STORE_BF16) launch_rows<GIST_STORE_BF16, GIST_STORE_E4M3, false>(st, a);
  else launch_rows<GIST_STORE_F16, GIST_STORE_E4M3, false>(st, a);
  return check_launch("quantize_rows");
}

size_t rms_norm_bwd_workspace(int64_t n, int d) {
  return static_cast<size_t>(bwd_blocks(n, d)) * static_cast<size_t>(d) * 4;
}

gist_status rms_norm_bwd(hipStream_t st, int64_t n, int d, const void* dy, int64_t lddy, int dy_store,
                         const void* h, int64_t ldh, int store, const float* gain, const float* rstd,
                         const void* dsum, int64_t ldds, const int32_t* labels, const int32_t* n_dev, void* dx, int64_t lddx,
                         float* dgain, void* ws) {
  if (n > 0) {
    const Bwd a{n, lddy, ldh, ldds, lddx, d, dy, h, gain, rstd, dsum, dx, dgain ? static_cast<float*>(ws) : nullptr,
                labels, n_dev};
    ProfScope ps(st, "rms_norm_bwd", 0.0,
                 static_cast<double>(n) * d *
                     (width_of(store) * (1.0 + (dsum && dx ? 1 : 0) + (dx ? 1 : 0)) + width_of(dy_store)));
    if (store == GIST_STORE_F32) launch_bwd_of<GIST_STORE_F32>(st, a, dy_store);
    else if (store == GIST_STORE_BF16) launch_bwd_of<GIST_STORE_BF16>(st, a, dy_store);
    else launch_bwd_of<GIST_STORE_F16>(st, a, dy_store);
    const gist_status s = check_launch("rms_norm_bwd");
    if (s != GIST_OK) return s;
  }
  if (dgain) {
    const int parts = n > 0 ? static_cast<int>(bwd_blocks(n, d)) : 0;
    ProfScope ps(st, "rms_norm_gain", 0.0, 4.0 * static_cast<double>(parts) * d);
    hipLaunchKernelGGL(gain_kernel, dim3(static_cast<unsigned>((d + 63) / 64)), dim3(64 * kJoinWaves), 0, st, parts, d,
                       static_cast<const float*>(ws), dgain);
    return check_launch("rms_norm_gain");
  }
  return GIST_OK;
}

}  // namespace gist
