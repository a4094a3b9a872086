// AdamW over many tensors in one launch, moments in fp32 or in 8 bits.
//
//   g = s dW,  m <- b1 m + (1 - b1) g,  v <- b2 v + (1 - b2) g^2,
//   W <- (1 - lr decay) W - a m / (sqrt(v) c + eps),   a = lr / (1 - b1^k), c = 1 / sqrt(1 - b2^k).
//
// 8-bit moments: m and sqrt(v) are held as e4m3 codes, 256 consecutive elements
// sharing an fp32 scale (the largest magnitude / 448); sqrt(v) because e4m3 then
// spans 2^35 of v.  A wave holds a block, four elements a lane, so the largest
// magnitude is one reduction and nothing is read twice.
// Rounding is stochastic: x / step + r, rounded down, r uniform on [0, 1).  v moves by
// 0.1% a step (b2 = 0.999) and half a step of e4m3 is up to 6%: rounded to the nearest,
// sqrt(v) would stay where it is until g^2 is a hundred times v, and would never fall.
// r comes from the element's index, the tensor's place in the list and a seed, so a
// step can be repeated bit for bit.  A sqrt(v) above zero is not rounded to zero: m over
// eps alone would be a step of any size.
//
// Bound by memory: 28 bytes an element in fp32, 16 with 8-bit moments, bf16 gradients and a bf16 copy.  A
// table of 131,072 x 1,024 and five more tensors in 8 bits: 731 us (3.25 GB, 4.45 TB/s).  A workgroup
// takes 1,024 elements; four times as many take 5 us longer of 95 (4,096 x 4,096, fp32 moments, bf16
// gradients) and are no better in the others.

#include "elem.cuh"

namespace gist {

namespace {

constexpr int kBlock = 256;
constexpr int kPiece = 4 * kBlock;      // elements of a workgroup
constexpr int kMostTensors = 40;        // of one launch: their addresses are kernel arguments (4 KB)
constexpr int64_t kMostGroups = int64_t{1} << 23;
constexpr float kTop = 448.f;           // largest e4m3 value
constexpr float kLeast = 0x1p-100f;     // a block whose largest magnitude is below this is zero

struct Tensor {
  float* W;
  const void* dW;
  void* m;
  void* v;
  float* ms;
  float* vs;
  void* copy;
  int64_t n;
  float decay;
  unsigned place;      // counts from 1
  int first;           // its first workgroup
  int8_t grad, copy_store, eight, pad;
};

struct Args {
  Tensor t[kMostTensors];
  const float* coef_dev;
  float step_size, inv_sqrt_bc2, lr, gscale, beta1, beta2, eps;
  unsigned seed;
  int fresh, count;
};
static_assert(sizeof(Args) <= 4096, "kernel arguments");

typedef unsigned u32u __attribute__((aligned(1)));

// A mixture of 32 bits: odd multipliers between shifts by about half the word
// (every step can be undone, so no two inputs meet).  Shifts and multipliers are those that
// C. Wellons found by search ("Prospecting for Hash Functions", 2018) to have the least bias.
__host__ __device__ __forceinline__ unsigned mix(unsigned x) {
  x ^= x >> 16;
  x *= 0x7feb352du;
  x ^= x >> 15;
  x *= 0x846ca68bu;
  return x ^ (x >> 16);
}

struct Coef {
  float step_size, inv_sqrt_bc2, gscale, beta1, omb1, beta2, omb2, eps, keep;
};

__device__ __forceinline__ void step_one(float& w, float g, float& m, float& v, const Coef& c) {
  g *= c.gscale;
  m = c.beta1 * m + c.omb1 * g;
  v = c.beta2 * v + c.omb2 * (g * g);
  w = c.keep * w - c.step_size * m / (sqrtf(v) * c.inv_sqrt_bc2 + c.eps);
}

// Four e4m3 codes from p on (the first `left` of them), times the block's scale.
__device__ __forceinline__ void load8(const void* base, int64_t e, int64_t left, float scale, float (&x)[4]) {
  const unsigned char* p = static_cast<const unsigned char*>(base) + e;
  unsigned u = 0;
  if (left >= 4) {
    u = *reinterpret_cast<const u32u*>(p);
  } else {
#pragma unroll
    for (int q = 0; q < 3; ++q)
      if (q < left) u |= static_cast<unsigned>(p[q]) << (8 * q);
  }
  x[0] = __builtin_amdgcn_cvt_f32_fp8(u, 0) * scale;
  x[1] = __builtin_amdgcn_cvt_f32_fp8(u, 1) * scale;
  x[2] = __builtin_amdgcn_cvt_f32_fp8(u, 2) * scale;
  x[3] = __builtin_amdgcn_cvt_f32_fp8(u, 3) * scale;
}

// Rounds the block's values (four a lane) and stores codes and scale.  r: 16 random bits each.
// A value that is not finite gets the code of NaN and leaves the others alone.
template <bool ROOT>
__device__ __forceinline__ void store8(void* base, int64_t e, int64_t left, float* scale, const float (&x)[4],
                                       const unsigned (&r)[4]) {
  float big = 0.f;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const float a = fabsf(x[q]);
    big = fmaxf(big, a < __builtin_inff() ? a : 0.f);
  }
  big = wave_max(big);
  const bool live = big >= kLeast;
  // k = floor(a / step + r), a = |x| (448 / big).  In 32 bits the sum is off by up to 4e-6 (a's three
  // roundings, times 16, and its own), which would put one code in 10^6 on the other side of a
  // border, and the block's next scale follows from the largest of them; so a wave with a sum within
  // 2^-17 of a whole number (one in 250) takes the sums again in 64.
  const float inv = live ? (1.f / big) * kTop : 0.f;
  float k[4], step[4];
  bool near = false;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const float a = fminf(fabsf(x[q]) * inv, kTop);
    const unsigned eb = max(__float_as_uint(a) >> 23, 121u);      // exponents below 2^-6 share its step
    step[q] = __uint_as_float((eb - 3u) << 23);
    const float t = fmaf(a, __uint_as_float((257u - eb) << 23), static_cast<float>(r[q]) * 0x1p-16f);
    near |= fabsf(t - rintf(t)) < 0x1p-17f;
    k[q] = floorf(t);
  }
  if (__any(near)) {
    const double inv64 = live ? (1.0 / static_cast<double>(big)) * static_cast<double>(kTop) : 0.0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const double a = fmin(static_cast<double>(fabsf(x[q])) * inv64, static_cast<double>(kTop));
      const int e = max(__double2hiint(a) >> 20, 1023 - 6);
      step[q] = __uint_as_float(static_cast<unsigned>(e - 1023 - 3 + 127) << 23);
      k[q] = static_cast<float>(floor(fma(a, __hiloint2double((2046 + 3 - e) << 20, 0), static_cast<double>(r[q]) * 0x1p-16)));
    }
  }
  float y[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if (ROOT && live && k[q] == 0.f && x[q] > 0.f) k[q] = 1.f;
    y[q] = copysignf(k[q] * step[q], x[q]);
    if (!(fabsf(x[q]) < __builtin_inff())) y[q] = __builtin_nanf("");
  }
  int u = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);   // exact: y are e4m3 values
  u = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], u, true);
  unsigned char* p = static_cast<unsigned char*>(base) + e;
  if (left >= 4) {
    *reinterpret_cast<u32u*>(p) = static_cast<unsigned>(u);
  } else {
#pragma unroll
    for (int q = 0; q < 3; ++q)
      if (q < left) p[q] = static_cast<unsigned char>(u >> (8 * q));
  }
  if ((threadIdx.x & 63) == 0) *scale = live ? big / kTop : 0.f;
}

template <int STORE>
__device__ __forceinline__ void load4(const void* base, int64_t e, int64_t left, float (&x)[4]) {
  if constexpr (STORE == GIST_STORE_F32) {
    load_some<STORE, 4>(base, e, left, 0.f, x);
  } else {
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
  }
}

template <int STORE>
__device__ __forceinline__ void store4(void* base, int64_t e, int64_t left, const float (&x)[4]) {
  typedef unsigned short us4 __attribute__((ext_vector_type(4), aligned(2)));
  unsigned short* p = static_cast<unsigned short*>(base) + e;
  us4 t;
#pragma unroll
  for (int q = 0; q < 4; ++q) t[q] = narrow<STORE>(x[q]);
  if (left >= 4) {
    *reinterpret_cast<us4*>(p) = t;
  } else {
#pragma unroll
    for (int q = 0; q < 3; ++q)
      if (q < left) p[q] = t[q];
  }
}

template <int GRAD, bool EIGHT>
__device__ __forceinline__ void piece(const Tensor& t, const Coef& c, int fresh, unsigned key, int64_t e0) {
  // a wave's 256 elements are one block: all of its lanes stay, for the reductions
  const int64_t e = e0 + 4 * static_cast<int64_t>(threadIdx.x), left = t.n - e;
  const int64_t blk = e >> 8;
  if ((blk << 8) >= t.n) return;     // the whole wave
  float w[4], g[4], m[4] = {}, v[4] = {};
  load4<GRAD>(t.dW, e, left, g);
  load_some<GIST_STORE_F32, 4>(t.W, e, left, 0.f, w);
  if (!fresh) {
    if constexpr (EIGHT) {
      load8(t.m, e, left, t.ms[blk], m);
      load8(t.v, e, left, t.vs[blk], v);
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] *= v[q];
    } else {
      load_some<GIST_STORE_F32, 4>(t.m, e, left, 0.f, m);
      load_some<GIST_STORE_F32, 4>(t.v, e, left, 0.f, v);
    }
  }
#pragma unroll
  for (int q = 0; q < 4; ++q) step_one(w[q], g[q], m[q], v[q], c);
  store_some<GIST_STORE_F32, 4>(t.W, e, left, w);
  if (t.copy) {
    if (t.copy_store == GIST_STORE_BF16) store4<GIST_STORE_BF16>(t.copy, e, left, w);
    else store4<GIST_STORE_F16>(t.copy, e, left, w);
  }
  if constexpr (EIGHT) {
    const unsigned x = static_cast<unsigned>(e) + key + static_cast<unsigned>(e >> 32) * 0x85ebca6bu;
    unsigned rm[4], rv[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const unsigned h = mix(x + q);
      rm[q] = h >> 16;
      rv[q] = h & 0xffffu;
      v[q] = q < left ? sqrtf(v[q]) : 0.f;
      m[q] = q < left ? m[q] : 0.f;
    }
    store8<false>(t.m, e, left, t.ms + blk, m, rm);
    store8<true>(t.v, e, left, t.vs + blk, v, rv);
  } else {
    store_some<GIST_STORE_F32, 4>(t.m, e, left, m);
    store_some<GIST_STORE_F32, 4>(t.v, e, left, v);
  }
}

__global__ __launch_bounds__(kBlock) void adamw_kernel(Args a) {
  // the workgroup's tensor: the last one whose first workgroup is not behind it
  const int b = blockIdx.x;
  int lo = 0, hi = a.count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.t[mid].first <= b) lo = mid;
    else hi = mid;
  }
  const Tensor t = a.t[lo];
  float lr = a.lr;
  unsigned seed = a.seed;
  Coef c{a.step_size, a.inv_sqrt_bc2, a.gscale, a.beta1, 1.f - a.beta1, a.beta2, 1.f - a.beta2, a.eps, 1.f};
  int fresh = a.fresh;
  if (a.coef_dev) {
    c.step_size = a.coef_dev[0];
    c.inv_sqrt_bc2 = a.coef_dev[1];
    fresh = a.coef_dev[2] != 0.f;
    lr = a.coef_dev[3];
    c.gscale = a.coef_dev[4];
    seed = __float_as_uint(a.coef_dev[5]);
  }
  c.keep = 1.f - lr * t.decay;
  const unsigned key = mix(seed ^ (t.place * 0x9e3779b9u));
  const int64_t e = static_cast<int64_t>(b - t.first) * kPiece;
  if (t.eight) {
    if (t.grad == GIST_STORE_F32) piece<GIST_STORE_F32, true>(t, c, fresh, key, e);
    else if (t.grad == GIST_STORE_BF16) piece<GIST_STORE_BF16, true>(t, c, fresh, key, e);
    else piece<GIST_STORE_F16, true>(t, c, fresh, key, e);
  } else {
    if (t.grad == GIST_STORE_F32) piece<GIST_STORE_F32, false>(t, c, fresh, key, e);
    else if (t.grad == GIST_STORE_BF16) piece<GIST_STORE_BF16, false>(t, c, fresh, key, e);
    else piece<GIST_STORE_F16, false>(t, c, fresh, key, e);
  }
}

}  // namespace

gist_status adamw(hipStream_t st, const gist_adamw_tensor* T, int64_t count, const float* coef, float beta1,
                  float beta2, float eps, const float* coef_dev) {
  Args a{};
  a.coef_dev = coef_dev;
  if (coef) {
    a.step_size = coef[0];
    a.inv_sqrt_bc2 = coef[1];
    a.fresh = coef[2] != 0.f;
    a.lr = coef[3];
    a.gscale = coef[4];
    a.seed = __builtin_bit_cast(unsigned, coef[5]);
  }
  a.beta1 = beta1;
  a.beta2 = beta2;
  a.eps = eps;
  for (int64_t i = 0; i < count;) {
    a.count = 0;
    int64_t groups = 0;
    double bytes = 0.0;
    while (i < count && a.count < kMostTensors) {
      const gist_adamw_tensor& s = T[i];
      const int64_t g = (s.n + kPiece - 1) / kPiece;
      if (g > 0) {
        if (groups + g > kMostGroups && a.count > 0) break;
        Tensor& t = a.t[a.count++];
        t.W = s.W;
        t.dW = s.dW;
        t.m = s.m;
        t.v = s.v;
        t.ms = s.m_scale;
        t.vs = s.v_scale;
        t.copy = s.copy;
        t.n = s.n;
        t.decay = s.weight_decay;
        t.place = static_cast<unsigned>(i + 1);
        t.first = static_cast<int>(groups);
        t.grad = static_cast<int8_t>(s.grad_store);
        t.copy_store = static_cast<int8_t>(s.copy_store);
        t.eight = s.m_scale != nullptr;
        groups += g;
        const double state = s.m_scale ? 2.0 + 8.0 / 256 : 8.0;
        bytes += s.n * (8.0 + (s.grad_store == GIST_STORE_F32 ? 4.0 : 2.0) + (a.fresh ? 1.0 : 2.0) * state +
                        (s.copy ? 2.0 : 0.0));
      }
      ++i;
    }
    if (a.count == 0) break;
    ProfScope ps(st, "adamw_update", 0.0, bytes);
    hipLaunchKernelGGL(adamw_kernel, dim3(static_cast<unsigned>(groups)), dim3(kBlock), 0, st, a);
    const gist_status s = check_launch("adamw_update");
    if (s != GIST_OK) return s;
  }
  return GIST_OK;
}

}  // namespace gist
