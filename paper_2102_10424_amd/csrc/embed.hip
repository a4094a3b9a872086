// Learned input rows: out[i] = scale table[ids[i]], and the table's gradient.
//
// The gradient adds the rows of dY whose ids are equal.  Adding them with
// floating-point atomics would make the sum's order, and its result, change
// from run to run, and would serialise a frequent id on one row; so the ids
// are sorted (stably, by a radix sort of (id, position)) and equal ids, now
// neighbours, are summed in position order: chunks of sorted positions in
// parallel, partial sums of ids that cross a chunk's border joined by a
// second kernel in chunk order.

#include <algorithm>

#include "elem.cuh"

namespace gist {

namespace {

constexpr int kBlock = 256;

// ---- lookup --------------------------------------------------------------------

// A group of 1 << tpr_log2 threads per row, V elements (16 bytes) a thread and
// step.  Bound by memory: 65,536 rows of 4,096 bf16 in 314 us (1.6 GB read and
// written, 5.1 TB/s); a call of 1,536 rows of 602 floats, 5.2 us, by its launch and
// the load of a row behind that of its id.
template <int STORE, int V>
__global__ __launch_bounds__(kBlock) void lookup_kernel(int n, int64_t V_rows, int d, int tpr_log2,
                                                        const void* __restrict__ table,
                                                        int64_t ldt, const int* __restrict__ ids,
                                                        float scale, float* __restrict__ out,
                                                        int64_t ldo) {
  const int lane = threadIdx.x & ((1 << tpr_log2) - 1);
  const int step = V << tpr_log2;
  for (int64_t row = (static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x) >> tpr_log2; row < n;
       row += (static_cast<int64_t>(gridDim.x) * kBlock) >> tpr_log2) {
    const int64_t id = ids[row];
    float* o = out + row * ldo;
    const bool in = id >= 0 && id < V_rows;
    const int64_t base = id * ldt;
    for (int j = V * lane; j < d; j += step) {
      float x[V] = {};
      if (in) load_some<STORE, V>(table, base + j, d - j, 0.f, x);
#pragma unroll
      for (int q = 0; q < V; ++q) x[q] *= scale;
      store_some<GIST_STORE_F32, V>(o, j, d - j, x);
    }
  }
}

// ---- sort -----------------------------------------------------------------------

constexpr int kDigit = 8, kBins = 1 << kDigit;
constexpr int kSortBlock = 1024, kItems = 2;   // threads, keys per thread and tile
constexpr int kTile = kSortBlock * kItems;     // 2,048

__device__ __forceinline__ int key_of(int id, int V) {   // padding sorts last
  return id >= 0 && id < V ? id : V;
}

// Where a tile's count of a digit lies: tile-major where the scatters add them up
// themselves, digit-major for the scan.
struct HistAt {
  int tiles;
  bool direct;
  __device__ __forceinline__ int64_t operator()(int64_t tile, int digit) const {
    return direct ? tile * kBins + digit : static_cast<int64_t>(digit) * tiles + tile;
  }
};

// Counts of every tile's digits.
template <bool FIRST>
__global__ __launch_bounds__(kSortBlock) void hist_kernel(int n, int V, const int* __restrict__ keys, int shift,
                                                          HistAt at, int* __restrict__ hist,
                                                          int* __restrict__ crossing) {
  __shared__ int cnt[kBins];
  if (FIRST && blockIdx.x == 0 && threadIdx.x < 2) crossing[threadIdx.x] = 0;
  if (threadIdx.x < kBins) cnt[threadIdx.x] = 0;
  __syncthreads();
  const int64_t base = static_cast<int64_t>(blockIdx.x) * kTile;
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    const int64_t e = base + i * kSortBlock + threadIdx.x;
    if (e < n) atomicAdd(&cnt[((FIRST ? key_of(keys[e], V) : keys[e]) >> shift) & (kBins - 1)], 1);
  }
  __syncthreads();
  if (threadIdx.x < kBins) hist[at(blockIdx.x, threadIdx.x)] = cnt[threadIdx.x];
}

// In-place exclusive scan of `count` ints (a multiple of 256) by one workgroup,
// 16 a thread and round.
__global__ __launch_bounds__(1024) void scan_kernel(int64_t count, int* __restrict__ v) {
  __shared__ int wsum[16];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  int carry = 0;
  for (int64_t base = 0; base < count; base += 16384) {
    const int64_t e = base + 16 * t;
    int4 x[4];
    int mine = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      x[q] = e < count ? reinterpret_cast<const int4*>(v + e)[q] : int4{0, 0, 0, 0};
      mine += x[q].x + x[q].y + x[q].z + x[q].w;
    }
    int inc = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int u = __shfl_up(inc, o, 64);
      if (lane >= o) inc += u;
    }
    if (lane == 63) wsum[wave] = inc;
    __syncthreads();
    int run = carry + inc - mine;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
      if (w < wave) run += wsum[w];
      carry += wsum[w];
    }
    if (e < count) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        int4 y;
        y.x = run;
        y.y = y.x + x[q].x;
        y.z = y.y + x[q].y;
        y.w = y.z + x[q].z;
        run = y.w + x[q].w;
        reinterpret_cast<int4*>(v + e)[q] = y;
      }
    }
    __syncthreads();   // wsum is read
  }
}

// Stable scatter of every tile's (key, position) pairs by one digit.  A wave
// holds kItems * 64 consecutive keys, 64 at a time; equal digits among a
// wave's 64 keys are found by matching the digit's bits with ballots.  Up to kDirect
// tiles each workgroup adds up the tiles' counts itself: one launch less than with the
// scan (two passes over 400,000 ids 31 us and 53, over 2,000,000 154 and 179).  Bound by
// launches and latency: 131,072 ids below 50,000 in 23 us.  (Adding the next digit's counts
// up on the way, with an atomic per wave and digit, made a pass one launch, of 18 us in
// place of 7.)
constexpr int kDirect = 1024;
template <bool FIRST>
__global__ __launch_bounds__(kSortBlock) void scatter_digit_kernel(
    int n, int V, const int* __restrict__ kin, const int* __restrict__ pin, int shift, HistAt at,
    const int* __restrict__ offs, int* __restrict__ kout, int* __restrict__ pout) {
  constexpr int kWaves = kSortBlock / 64, kQ = kSortBlock / kBins;
  __shared__ int cnt[kWaves][kBins];
  __shared__ int sums[kQ][2][kBins];
  __shared__ int wsum[kBins / 64];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  for (int x = t; x < kWaves * kBins; x += kSortBlock) (&cnt[0][0])[x] = 0;
  if (at.direct) {   // thread t: digit t mod kBins, every kQ-th tile
    const int dg = t & (kBins - 1), part = t / kBins;
    int total = 0, before = 0;
#pragma unroll 16
    for (int x = part; x < at.tiles; x += kQ) {
      const int c = offs[x * kBins + dg];
      total += c;
      before += x < static_cast<int>(blockIdx.x) ? c : 0;
    }
    sums[part][0][dg] = total;
    sums[part][1][dg] = before;
  }
  const int64_t base = static_cast<int64_t>(blockIdx.x) * kTile + wave * (kItems * 64);
  int key[kItems], rank[kItems];
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    const int64_t e = base + i * 64 + lane;
    key[i] = e < n ? (FIRST ? key_of(kin[e], V) : kin[e]) : 0;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    const bool in = base + i * 64 + lane < n;
    const int dg = (key[i] >> shift) & (kBins - 1);
    unsigned long long m = __ballot(in);
#pragma unroll
    for (int b = 0; b < kDigit; ++b) {
      const unsigned long long s = __ballot((dg >> b) & 1);
      m &= (dg >> b) & 1 ? s : ~s;
    }
    const int before = __popcll(m & ((1ull << lane) - 1));
    const int had = cnt[wave][dg];   // the wave's keys of this digit so far
    rank[i] = had + before;
    wave_sync();
    if (in && before == 0) cnt[wave][dg] = had + __popcll(m);
    wave_sync();
  }
  int first = 0, total = 0, inc = 0;   // digit t: its keys' first place in the tile
  if (t < kBins) {
    if (at.direct) {
#pragma unroll
      for (int x = 0; x < kQ; ++x) {
        total += sums[x][0][t];
        first += sums[x][1][t];
      }
      inc = total;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(inc, o, 64);
        if (lane >= o) inc += u;
      }
      if (lane == 63) wsum[wave] = inc;
    } else {
      first = offs[at(blockIdx.x, t)];
    }
  }
  __syncthreads();
  if (t < kBins) {
    if (at.direct) {
      first += inc - total;
      for (int w = 0; w < wave; ++w) first += wsum[w];
    }
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {   // the waves' first places
      const int c = cnt[w][t];
      cnt[w][t] = first;
      first += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    const int64_t e = base + i * 64 + lane;
    if (e < n) {
      const int to = cnt[wave][(key[i] >> shift) & (kBins - 1)] + rank[i];
      kout[to] = key[i];
      pout[to] = FIRST ? static_cast<int>(e) : pin[e];
    }
  }
}

// Up to kSmall ids: the whole sort in one workgroup, keys and positions in
// registers and, between two digits, in LDS.  Ids that ascend already (the node
// map of a cluster mini-batch) are only copied.  The SGD step of 1,630 such rows of
// 100 columns takes 11.8 us in three launches; 60.7 with three passes of three kernels.
constexpr int kSmallThreads = 1024, kSmallItems = 8, kSmall = kSmallThreads * kSmallItems;
__global__ __launch_bounds__(kSmallThreads) void small_sort_kernel(int n, int V, const int* __restrict__ ids,
                                                                   int passes, int* __restrict__ keys,
                                                                   int* __restrict__ pos,
                                                                   int* __restrict__ crossing) {
  constexpr int kWaves = kSmallThreads / 64;
  __shared__ int cnt[kWaves][kBins];
  __shared__ int lk[kSmall], lp[kSmall];
  __shared__ int wsum[kBins / 64];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int items = (n + kSmallThreads - 1) / kSmallThreads;   // of 64 keys per wave
  const int base = wave * items * 64;
  int key[kSmallItems], ps[kSmallItems];
  int down = 0;
  if (t < 2) crossing[t] = 0;
#pragma unroll
  for (int i = 0; i < kSmallItems; ++i) {
    const int e = base + i * 64 + lane;
    key[i] = V;
    ps[i] = e;
    if (i < items && e < n) {
      key[i] = key_of(ids[e], V);
      if (e > 0) down |= key_of(ids[e - 1], V) > key[i];
    }
  }
  if (!__syncthreads_or(down)) passes = 0;
  for (int p = 0; p < passes; ++p) {
    const int shift = p * kDigit;
    for (int x = t; x < kWaves * kBins; x += kSmallThreads) (&cnt[0][0])[x] = 0;
    __syncthreads();
    int rank[kSmallItems];
#pragma unroll
    for (int i = 0; i < kSmallItems; ++i) {
      if (i >= items) break;
      const bool in = base + i * 64 + lane < n;
      const int dg = (key[i] >> shift) & (kBins - 1);
      unsigned long long m = __ballot(in);
#pragma unroll
      for (int b = 0; b < kDigit; ++b) {
        const unsigned long long s = __ballot((dg >> b) & 1);
        m &= (dg >> b) & 1 ? s : ~s;
      }
      const int before = __popcll(m & ((1ull << lane) - 1));
      const int had = cnt[wave][dg];
      rank[i] = had + before;
      wave_sync();
      if (in && before == 0) cnt[wave][dg] = had + __popcll(m);
      wave_sync();
    }
    __syncthreads();
    int total = 0, inc = 0;
    if (t < kBins) {   // digit t: keys of all waves, then of the digits before it
      for (int w = 0; w < kWaves; ++w) {
        const int c = cnt[w][t];
        cnt[w][t] = total;
        total += c;
      }
      inc = total;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(inc, o, 64);
        if (lane >= o) inc += u;
      }
      if (lane == 63) wsum[wave] = inc;
    }
    __syncthreads();
    if (t < kBins) {
      int start = inc - total;
      for (int w = 0; w < wave; ++w) start += wsum[w];
      for (int w = 0; w < kWaves; ++w) cnt[w][t] += start;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSmallItems; ++i) {
      if (i >= items) break;
      if (base + i * 64 + lane < n) {
        const int to = cnt[wave][(key[i] >> shift) & (kBins - 1)] + rank[i];
        lk[to] = key[i];
        lp[to] = ps[i];
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSmallItems; ++i) {
      if (i >= items) break;
      const int e = base + i * 64 + lane;
      if (e < n) {
        key[i] = lk[e];
        ps[i] = lp[e];
      }
    }
  }
#pragma unroll
  for (int i = 0; i < kSmallItems; ++i) {
    const int e = base + i * 64 + lane;
    if (i < items && e < n) {
      keys[e] = key[i];
      pos[e] = ps[i];
    }
  }
}

// ---- sums over equal ids -----------------------------------------------------------

constexpr int kV = 4;   // columns per thread

// A row's finished sum: the dense gradient, or the SGD step on the table's row `t`.
template <bool SGD>
__device__ __forceinline__ void finish(float* p, int left, const float (&acc)[kV], const float (&t)[kV], float scale,
                                       float lr) {
  float x[kV];
#pragma unroll
  for (int q = 0; q < kV; ++q) x[q] = SGD ? fmaf(-lr, scale * acc[q], t[q]) : scale * acc[q];
  store_some<GIST_STORE_F32, kV>(p, 0, left, x);
}

// Lanes (their logarithm) that zero a row's `width` columns together.
__host__ __device__ __forceinline__ int zero_lanes_log2(int width) {
  int l = 0;
  while (l < 6 && (kV << l) < width) ++l;
  return l;
}

// Zero rows that no id names (dense gradient), columns j0 .. j1 - 1: a wave per
// 1 << rows_log2 rows, each lane looking its row up in the sorted ids.  Writing them
// here, and not all rows before the sums, leaves each row one write.
__device__ __forceinline__ void zero_rows(int n, int Vn, int j0, int j1, int rows_log2, int64_t wave,
                                          const int* __restrict__ keys, float* __restrict__ out,
                                          int64_t ldo) {
  const int lane = threadIdx.x & 63, R = 1 << rows_log2;
  const int64_t r0 = wave << rows_log2;
  if (r0 >= Vn) return;
  const int64_t r = r0 + (lane & (R - 1));
  int lo = 0, hi = n;
  while (lo < hi) {
    const int mid = lo + ((hi - lo) >> 1);
    if (keys[mid] < r) lo = mid + 1;
    else hi = mid;
  }
  const unsigned long long m = __ballot(r < Vn && (lo >= n || keys[lo] != r));
  const int tl = zero_lanes_log2(j1 - j0), l = lane & ((1 << tl) - 1);
  const float z[kV] = {};
  for (int q = lane >> tl; q < R; q += 64 >> tl)
    if (m >> q & 1)
      for (int j = j0 + kV * l; j < j1; j += kV << tl) store_some<GIST_STORE_F32, kV>(out + (r0 + q) * ldo, j, j1 - j, z);
}

// Chunks of `len` sorted positions (a multiple of kBatch), one group of threads
// each (n + len - 1 fits int32: the caller refuses more than 2^31 - 128 ids); blockIdx.y: slab of columns.  part[2 c] is the sum of chunk c's first id
// where that id began in an earlier chunk, part[2 c + 1] that of its last id where
// it began in this chunk and goes on in the next.  The chunks with such an id are
// listed, in no order: crossing[0] of them, from crossing[2] on, and crossing[1] with
// an id of more than kFew parts, from crossing[1 + chunks] down.  Rows are loaded kBatch
// at a time and added in order.  Bound by memory: 131,072 rows of 1,024 columns in
// 150 us (537 MB of rows, 4.5 TB/s with results and parts).
constexpr int kFew = 16;
constexpr int kBatch = 8;
// Dense: the blocks behind the chunks' (from blockIdx.x == sums on) zero the other rows,
// 164 us together for a table of 50,000 rows, where a launch of their own took 24 beside
// 152; and 8 ids of a table of 1,063 x 563 take 10.5 us, 31 with that launch, in which 17
// waves zeroed 64 rows each.
template <bool SGD>
__global__ __launch_bounds__(kBlock) void sum_kernel(int sums, int rows_log2, int n, int Vn, int d, int tpr_log2, int len,
                                                     const int* __restrict__ keys,
                                                     const int* __restrict__ pos, float scale,
                                                     const float* __restrict__ dY, int64_t ldy,
                                                     float lr, float* __restrict__ out,
                                                     int64_t ldo, float* __restrict__ part,
                                                     int64_t ldp, int* __restrict__ crossing) {
  if (!SGD && blockIdx.x >= sums) {
    const int j0 = (kV * static_cast<int>(blockIdx.y)) << tpr_log2;
    zero_rows(n, Vn, j0, min(d, j0 + (kV << tpr_log2)), rows_log2,
              (static_cast<int64_t>(blockIdx.x - sums) * kBlock + threadIdx.x) >> 6, keys, out, ldo);
    return;
  }
  const int lane = threadIdx.x & ((1 << tpr_log2) - 1);
  const int64_t c = (static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x) >> tpr_log2;
  const int64_t b64 = c * len;
  if (b64 >= n) return;
  const int b = static_cast<int>(b64), e = static_cast<int>(min<int64_t>(n, b64 + len));
  const int j = kV * (lane + (static_cast<int>(blockIdx.y) << tpr_log2));
  if (j >= d) return;
  int cur = keys[b];
  if (cur == Vn) return;   // padding only
  bool head = b > 0 && keys[b - 1] == cur;
  float acc[kV] = {}, old[kV];   // the sum of cur's rows, and its row of the table
  if (SGD) load_some<GIST_STORE_F32, kV>(out + cur * ldo + j, 0, d - j, 0.f, old);
  for (int i = b; i < e; i += kBatch) {
    int k[kBatch], p[kBatch];
    float x[kBatch][kV], o[kBatch][kV];
    // the arrays are padded to whole batches
#pragma unroll
    for (int u = 0; u < kBatch; u += 4) {
      const int4 kk = *reinterpret_cast<const int4*>(keys + i + u), pp = *reinterpret_cast<const int4*>(pos + i + u);
      k[u] = kk.x; k[u + 1] = kk.y; k[u + 2] = kk.z; k[u + 3] = kk.w;
      p[u] = pp.x; p[u + 1] = pp.y; p[u + 2] = pp.z; p[u + 3] = pp.w;
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
      if (i + u < e && k[u] != Vn) {
        load_some<GIST_STORE_F32, kV>(dY, p[u] * ldy + j, d - j, 0.f, x[u]);
        // The table rows of ids that begin here, all on their way before the first is needed:
        // 131,072 ids of 64 columns 32 us, 40 with each loaded when its sum was done.
        if (SGD && k[u] != (u ? k[u - 1] : cur)) load_some<GIST_STORE_F32, kV>(out + k[u] * ldo + j, 0, d - j, 0.f, o[u]);
      }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      if (i + u >= e) break;
      if (k[u] != cur) {
        if (head) store_vec<kV>(part + 2 * c * ldp + j, acc);
        else finish<SGD>(out + cur * ldo + j, d - j, acc, old, scale, lr);
        head = false;
        cur = k[u];
        if (SGD) {
#pragma unroll
          for (int q = 0; q < kV; ++q) old[q] = o[u][q];
        }
#pragma unroll
        for (int q = 0; q < kV; ++q) acc[q] = 0.f;
        if (cur == Vn) return;
      }
#pragma unroll
      for (int q = 0; q < kV; ++q) acc[q] += x[u][q];
    }
  }
  if (head) store_vec<kV>(part + 2 * c * ldp + j, acc);
  else if (e < n && keys[e] == cur) {
    store_vec<kV>(part + (2 * c + 1) * ldp + j, acc);
    if (j == 0) {
      const int64_t far = b64 + static_cast<int64_t>(kFew) * len;   // the id's part kFew begins here
      if (far < n && keys[far] == cur) crossing[1 + (n + len - 1) / len - atomicAdd(crossing + 1, 1)] = static_cast<int>(c);
      else crossing[2 + atomicAdd(crossing, 1)] = static_cast<int>(c);
    }
  } else finish<SGD>(out + cur * ldo + j, d - j, acc, old, scale, lr);
}

// Ids that cross chunk borders: the parts of a listed chunk's id are added in chunk
// order.  Most have two or three parts and take a group of threads each.  A
// frequent id takes a workgroup per 128 columns, 32 groups of 32 threads, each
// adding a run of the parts, and then the runs' sums in order.  (131,072 ids of
// 50,000 by a power law, 1,024 columns: 25 us with a group per id, whose longest, 262
// parts, took that long; 16 so.)
constexpr int kJoinThreads = 1024, kJoinBlocks = 256, kSlabLog2 = 5;

// Sum of parts x0 .. x1 - 1 of the id that begins in chunk c (part 0 is that
// chunk's second), column j.
__device__ __forceinline__ void add_parts(const float* part, int64_t ldp, int64_t c, int64_t x0, int64_t x1, int j,
                                          float (&acc)[kV]) {
  for (int64_t x = x0; x < x1; x += kBatch) {
    float y[kBatch][kV];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int64_t i = min(x + u, x1 - 1);
      load_vec<GIST_STORE_F32, kV>(part, (2 * (c + i) + (i == 0)) * ldp + j, y[u]);
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
      if (x + u < x1) {
#pragma unroll
        for (int q = 0; q < kV; ++q) acc[q] += y[u][q];
      }
  }
}

template <bool SGD>
__global__ __launch_bounds__(kJoinThreads) void join_kernel(int n, int d, int tpr_log2, int len,
                                                            const int* __restrict__ keys, float scale,
                                                            float lr, float* __restrict__ out,
                                                            int64_t ldo, const float* __restrict__ part,
                                                            int64_t ldp, const int* __restrict__ crossing) {
  __shared__ float sh[kJoinThreads][kV];
  const int t = threadIdx.x, chunks = (n + len - 1) / len;
  // chunk x begins with the id (then all of the chunk before it, from c + 1 on, is the id's)
  auto begins = [&](int64_t x, int cur) { return x * len < n && keys[x * len] == cur; };
  if (blockIdx.x >= kJoinBlocks) {   // ids of few parts
    const int lane = t & ((1 << tpr_log2) - 1), groups = kJoinThreads >> tpr_log2, listed = crossing[0];
    const int blocks = gridDim.x - kJoinBlocks;
    // neighbouring items to different workgroups: with narrow rows a few could take them all
    for (int it = (t >> tpr_log2) * blocks + (blockIdx.x - kJoinBlocks); it < listed; it += blocks * groups) {
      const int64_t c = crossing[2 + it];
      const int cur = keys[(c + 1) * len];
      int count = 2;
#pragma unroll
      for (int x = 2; x < kFew; ++x) count += begins(c + x, cur);
      for (int j = kV * lane; j < d; j += kV << tpr_log2) {
        float acc[kV] = {}, old[kV];
        if (SGD) load_some<GIST_STORE_F32, kV>(out + cur * ldo + j, 0, d - j, 0.f, old);
        add_parts(part, ldp, c, 0, count, j, acc);
        finish<SGD>(out + cur * ldo + j, d - j, acc, old, scale, lr);
      }
    }
    return;
  }
  constexpr int kGroups = kJoinThreads >> kSlabLog2, kSlab = kV << kSlabLog2;
  const int lane = t & ((1 << kSlabLog2) - 1), grp = t >> kSlabLog2;
  const int slabs = (d + kSlab - 1) / kSlab;
  const int64_t units = static_cast<int64_t>(crossing[1]) * slabs;
  for (int64_t it = blockIdx.x; it < units; it += kJoinBlocks) {
    const int64_t c = crossing[1 + chunks - it / slabs];
    const int j = static_cast<int>(it % slabs) * kSlab + kV * lane;
    const int cur = keys[(c + 1) * len];
    int64_t count = 1;
    for (int64_t x = c + 1;; x += kJoinThreads) {
      const int more = __syncthreads_count(begins(x + t, cur));   // and sh is read
      count += more;
      if (more < kJoinThreads) break;
    }
    const int64_t run = (count + kGroups - 1) / kGroups;
    const int64_t x0 = min<int64_t>(count, grp * run), x1 = min<int64_t>(count, x0 + run);
    float acc[kV] = {};
    if (j < d) add_parts(part, ldp, c, x0, x1, j, acc);
#pragma unroll
    for (int q = 0; q < kV; ++q) sh[t][q] = acc[q];
    __syncthreads();
    if (grp == 0 && j < d) {
      for (int g = 1; g < kGroups && g * run < count; ++g)
#pragma unroll
        for (int q = 0; q < kV; ++q) acc[q] += sh[(g << kSlabLog2) + lane][q];
      float old[kV];
      if (SGD) load_some<GIST_STORE_F32, kV>(out + cur * ldo + j, 0, d - j, 0.f, old);
      finish<SGD>(out + cur * ldo + j, d - j, acc, old, scale, lr);
    }
  }
}

size_t up256(size_t x) { return (x + 255) & ~size_t(255); }

// Threads (their logarithm) that a row's sum takes.
int group_log2(int d) { return std::min(8, ceil_log2((d + kV - 1) / kV)); }

struct GradPlan {
  int64_t tiles, chunks, ldp;
  int len, passes;
  size_t keys, hist, part, cross;
  size_t total() const { return 4 * keys + hist + part + cross; }
};

GradPlan plan(int64_t n, int64_t V, int d) {
  GradPlan p;
  p.tiles = (n + kTile - 1) / kTile;
  p.passes = (ceil_log2(V + 1) + kDigit - 1) / kDigit;
  // short chunks where there are few rows, or narrow ones (a group of few threads each), so
  // that there are enough groups; parts cost two rows a chunk.  (131,072 ids: one column 12 us
  // with chunks of 8, 23 of 32; 32 columns 35 and 34, 64 columns 60 and 40; 2,000,000 ids of one
  // column 66 with chunks of 32, 100 of 128.)  One chunk, which needs no
  // join, for up to 32 ids.
  const int tl = group_log2(d);
  const int64_t most8 = std::max<int64_t>(32768, (int64_t{1} << 20) >> tl);
  const int64_t most32 = std::max<int64_t>(1 << 20, (int64_t{1} << 23) >> tl);
  p.len = n <= 32 ? 32 : n <= most8 ? kBatch : n <= most32 ? 32 : 128;
  p.chunks = (n + p.len - 1) / p.len;
  p.ldp = (d + 3) / 4 * 4;
  p.keys = up256(static_cast<size_t>(n) * 4);
  p.hist = up256(static_cast<size_t>(p.tiles) * kBins * 4);
  // room for the chunks of any smaller n too: a workspace for n ids serves fewer
  const int64_t room = std::max<int64_t>(p.chunks, n > most32 ? most32 / 32 : n > most8 ? most8 / kBatch : 0);
  p.part = up256(static_cast<size_t>(room) * 2 * p.ldp * 4);
  p.cross = n > 0 ? up256(static_cast<size_t>(room + 2) * 4) : 0;
  return p;
}

}  // namespace

gist_status embed_lookup(hipStream_t st, int64_t n, int64_t V, int d, const void* table,
                         int64_t ldt, int store, const int32_t* ids, float scale, float* out,
                         int64_t ldo) {
  const int eb = store == GIST_STORE_F32 ? 4 : 2, v = store == GIST_STORE_F32 ? 4 : 8;
  const int tl = std::min(8, ceil_log2((d + v - 1) / v));
  const int64_t blocks = std::min<int64_t>(((n << tl) + kBlock - 1) / kBlock, 1 << 22);
  ProfScope ps(st, "embed_lookup", static_cast<double>(n) * d,
               4.0 * n + static_cast<double>(n) * d * (eb + 4));
#define LOOKUP(S, W)                                                                         \
  lookup_kernel<S, W><<<dim3(static_cast<unsigned>(blocks)), kBlock, 0, st>>>(               \
      static_cast<int>(n), V, d, tl, table, ldt, ids, scale, out, ldo)
  if (store == GIST_STORE_F32) LOOKUP(GIST_STORE_F32, 4);
  else if (store == GIST_STORE_BF16) LOOKUP(GIST_STORE_BF16, 8);
  else LOOKUP(GIST_STORE_F16, 8);
#undef LOOKUP
  return check_launch("embed_lookup");
}

size_t embed_grad_workspace(int64_t n, int64_t V, int d) { return plan(n, V, d).total(); }

gist_status embed_grad(hipStream_t st, int64_t n, int64_t V, int d, const int32_t* ids,
                       float scale, const float* dY, int64_t ldy, bool sgd, float lr, float* out,
                       int64_t ldo, void* ws) {
  const GradPlan p = plan(n, V, d);
  const int tl = group_log2(d);
  const int slabs = (d + (kV << tl) - 1) / (kV << tl);
  const int64_t sums = ((p.chunks << tl) + kBlock - 1) / kBlock;
  // rows to be zeroed per wave: 64, fewer where that leaves the card short of waves, and not
  // fewer than a wave's lanes reach at once
  int rl = 6;
  while (rl > 0 && (V >> rl) * slabs < 4096) --rl;
  rl = std::max(rl, 6 - zero_lanes_log2(std::min(d, kV << tl)));
  const int64_t zeros = sgd ? 0 : (((V + (1 << rl) - 1) >> rl) * 64 + kBlock - 1) / kBlock;
  if ((sums + zeros) * kBlock >= int64_t{1} << 32)
    return set_error(GIST_E_UNSUPPORTED, "embed_grad: n * d or V exceeds the grid");
  char* c = static_cast<char*>(ws);
  int* k[2] = {reinterpret_cast<int*>(c), reinterpret_cast<int*>(c + p.keys)};
  int* q[2] = {reinterpret_cast<int*>(c + 2 * p.keys), reinterpret_cast<int*>(c + 3 * p.keys)};
  int* hist = reinterpret_cast<int*>(c + 4 * p.keys);
  float* part = reinterpret_cast<float*>(c + 4 * p.keys + p.hist);
  int* cross = reinterpret_cast<int*>(c + 4 * p.keys + p.hist + p.part);
  const int ni = static_cast<int>(n), vi = static_cast<int>(V), tiles = static_cast<int>(p.tiles);
  int cur = 0;
  if (n > 0 && n <= kSmall) {
    ProfScope ps(st, "embed_sort_small", 0.0, 12.0 * n);
    small_sort_kernel<<<1, kSmallThreads, 0, st>>>(ni, vi, ids, p.passes, k[0], q[0], cross);
  } else if (n > 0) {
    ProfScope ps(st, "embed_sort", 0.0, 8.0 * n * p.passes);
    const HistAt at{tiles, tiles <= kDirect};
    const dim3 g(static_cast<unsigned>(tiles));
    for (int i = 0; i < p.passes; ++i) {
      const int *const kin = i == 0 ? ids : k[cur ^ 1], *const pin = i == 0 ? nullptr : q[cur ^ 1];
      const int shift = i * kDigit;
      if (i == 0) hist_kernel<true><<<g, kSortBlock, 0, st>>>(ni, vi, kin, shift, at, hist, cross);
      else hist_kernel<false><<<g, kSortBlock, 0, st>>>(ni, vi, kin, shift, at, hist, cross);
      if (!at.direct) scan_kernel<<<1, 1024, 0, st>>>(p.tiles * kBins, hist);
      if (i == 0) scatter_digit_kernel<true><<<g, kSortBlock, 0, st>>>(ni, vi, kin, pin, shift, at, hist, k[cur], q[cur]);
      else scatter_digit_kernel<false><<<g, kSortBlock, 0, st>>>(ni, vi, kin, pin, shift, at, hist, k[cur], q[cur]);
      cur ^= 1;
    }
    cur ^= 1;
  }
  if (sums + zeros > 0) {
    ProfScope ps(st, "embed_sum", static_cast<double>(n) * d, 4.0 * d * (2.0 * n + (sgd ? n : V)));
    const dim3 g(static_cast<unsigned>(sums + zeros), static_cast<unsigned>(slabs));
    const int first = static_cast<int>(sums);
    if (sgd)
      sum_kernel<true><<<g, kBlock, 0, st>>>(first, rl, ni, vi, d, tl, p.len, k[cur], q[cur], scale, dY, ldy, lr, out,
                                             ldo, part, p.ldp, cross);
    else
      sum_kernel<false><<<g, kBlock, 0, st>>>(first, rl, ni, vi, d, tl, p.len, k[cur], q[cur], scale, dY, ldy, lr, out,
                                              ldo, part, p.ldp, cross);
  }
  if (p.chunks > 1) {
    ProfScope ps(st, "embed_join", 0.0, 0.0);
    const dim3 gj(2 * kJoinBlocks);   // 1,024 threads each: two a CU
    if (sgd) join_kernel<true><<<gj, kJoinThreads, 0, st>>>(ni, d, tl, p.len, k[cur], scale, lr, out, ldo, part, p.ldp, cross);
    else join_kernel<false><<<gj, kJoinThreads, 0, st>>>(ni, d, tl, p.len, k[cur], scale, lr, out, ldo, part, p.ldp, cross);
  }
  return check_launch("embed_grad");
}

}  // namespace gist
