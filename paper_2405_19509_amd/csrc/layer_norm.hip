// Layer norm and its gradients, those of its weights per chunk.
//
// All of it is memory traffic (22 operations per value at most against 6 to 20 bytes), so a row is read
// once: a block holds it in registers, NV vectors of 16 bytes a thread, from the first sum to the result.
// Rows start anywhere (vector loads need no alignment here); only a row's last vector is taken apart.
// Rows longer than the registers of 1024 threads (kMostUnits) go through memory again for each sum.  The gradients
// of bf16 rows of 16385 to 32768 values do not fit them either: with four vectors a thread 172 registers are spilled (1620
// rows of 20000 250 to 300 us against 41 for the bytes; rows of 40000, through memory again, 86).
//
// Gradients: a block takes a run of rows of one chunk and keeps its columns' sums of dy h and dy in
// registers; runs are joined by a second kernel where a chunk has more than one.
#include "common.h"
#include "head.h"

namespace gcx {
namespace {

constexpr int kThreads = 256;

template <typename T>
constexpr int kUnit = 16 / int(sizeof(T));

// 16 bytes of a row in registers, as words (vectors of bf16 would take a register each); values past
// a row's end (`left` of the U exist) are neither read nor written, and zero.
template <typename T>
struct Unit {
  static constexpr int U = kUnit<T>;
  typedef uint32_t Words __attribute__((ext_vector_type(4)));
  typedef uint32_t Anywhere __attribute__((ext_vector_type(4), aligned(2)));
  Words w;
  __device__ __forceinline__ void load(const T *at, int left) {
    if (left >= U) {
      w = *reinterpret_cast<const Anywhere *>(at);
    } else {
      w = Words{0, 0, 0, 0};
#pragma unroll
      for (int e = 0; e < U; ++e)
        if (e < left) {
          if constexpr (U == 8)
            w[e / 2] |= uint32_t(__builtin_bit_cast(uint16_t, at[e])) << (e % 2 * 16);
          else
            w[e] = __builtin_bit_cast(uint32_t, at[e]);
        }
    }
  }
  // past a row's end its first value again: what is made of it there is as finite as the row's own
  __device__ __forceinline__ void fill(int left) {
    if (left > 0 && left < U) {
      const uint32_t first = U == 8 ? (w[0] & 0xffffu) * 0x10001u : w[0];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if constexpr (U == 8) {
          if (2 * k >= left)
            w[k] = first;
          else if (2 * k + 1 == left)
            w[k] |= first << 16;
        } else {
          if (k >= left) w[k] = first;
        }
      }
    }
  }
  __device__ __forceinline__ float operator[](int e) const {
    if constexpr (U == 8)
      return __uint_as_float(e % 2 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
    else
      return __uint_as_float(w[e]);
  }
  template <class V>
  __device__ __forceinline__ void set(int q, V value) {  // values 4 q .. 4 q + 3
    typedef __bf16 Pair __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int k = q * 16 / U; k < (q + 1) * 16 / U; ++k) {
      if constexpr (U == 8)
        w[k] = __builtin_bit_cast(uint32_t, Pair{static_cast<__bf16>(value(2 * k)), static_cast<__bf16>(value(2 * k + 1))});
      else
        w[k] = __float_as_uint(value(k));
    }
  }
  // what was made of the values so far is made anew from here on, and not held in registers
  __device__ __forceinline__ void forget() { asm volatile("" : "+v"(w)); }
  __device__ __forceinline__ void store(T *at, int left) const {
    if (left >= U) {
      *reinterpret_cast<Anywhere *>(at) = w;
    } else {
#pragma unroll
      for (int e = 0; e < U; ++e)
        if (e < left) {
          if constexpr (U == 8)
            at[e] = __builtin_bit_cast(__bf16, uint16_t(w[e / 2] >> (e % 2 * 16)));
          else
            at[e] = __uint_as_float(w[e]);
        }
    }
  }
};

template <int U>
__device__ __forceinline__ void load_floats(const float *at, int left, float (&v)[U]) {
  typedef float Vec __attribute__((ext_vector_type(4), aligned(4)));
  if (left >= U) {
#pragma unroll
    for (int e = 0; e < U; ++e) v[e] = reinterpret_cast<const Vec *>(at)[e / 4][e % 4];
  } else {
#pragma unroll
    for (int e = 0; e < U; ++e) v[e] = e < left ? at[e] : 0.f;
  }
}
template <int U>
__device__ __forceinline__ void store_floats(float *at, int left, const float (&v)[U]) {
  typedef float Vec __attribute__((ext_vector_type(4), aligned(4)));
  if (left >= U) {
#pragma unroll
    for (int q = 0; q < U / 4; ++q) reinterpret_cast<Vec *>(at)[q] = Vec{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
  } else {
#pragma unroll
    for (int e = 0; e < U; ++e)
      if (e < left) at[e] = v[e];
  }
}

// Sum over a wave, the same in every lane: neighbours, pairs, .. of a row of 16 lanes, then the rows, in the
// vector unit's own lane moves (a row's time is in this chain: with LDS shuffles 733 us for 25,600 rows of 16384 bf16, so 545)
__device__ __forceinline__ float wave_total(float v) {
#define GCX_ADD(ctrl, rows) \
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ctrl, rows, 0xf, true))
  GCX_ADD(0x111, 0xf);  // from one lane before, two, four, eight
  GCX_ADD(0x112, 0xf);
  GCX_ADD(0x114, 0xf);
  GCX_ADD(0x118, 0xf);
  GCX_ADD(0x142, 0xa);  // lane 15 of the row before, into rows 1 and 3
  GCX_ADD(0x143, 0xc);  // lane 31, into rows 2 and 3
#undef GCX_ADD
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), kWave - 1));
}

// Sums of K values over a block of up to MOST threads, in one order.  `turn` alternates from call to call, so
// that one barrier is enough; waves that a block does not have count as zeros, which start() lays down.
template <int MOST, int K>
struct BlockSums {
  static constexpr int kWaves = MOST / kWave;
  typedef float Row[2][kWaves][K];
  __device__ static __forceinline__ void start(Row &part) {
    if constexpr (kWaves > 1) {
      for (int e = threadIdx.x; e < 2 * kWaves * K; e += blockDim.x) (&part[0][0][0])[e] = 0.f;
      __syncthreads();
    }
  }
  __device__ static __forceinline__ void sum(Row &part, float (&v)[K], int turn) {
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = wave_total(v[k]);
    if constexpr (kWaves > 1) {
      if (threadIdx.x % kWave == 0)
#pragma unroll
        for (int k = 0; k < K; ++k) part[turn][threadIdx.x / kWave][k] = v[k];
      __syncthreads();
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w)
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] += part[turn][w][k];
    }
  }
};

// Rows of up to NV units a thread, in registers; a block's next row on its way while it works on one.
template <typename T, int MOST, int NV>
__global__ __launch_bounds__(MOST) void norm_kernel(const T *x, const float *gamma, const float *beta, int64_t rows,
                                                       int64_t d, float eps, T *y, float *mean, float *rstd) {
  constexpr int U = kUnit<T>;
  float g[NV][U], b[NV][U];
  uint32_t c[NV];  // columns
  int left[NV];    // how many of a unit's there are
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    c[i] = (i * blockDim.x + threadIdx.x) * U;
    left[i] = d - c[i] < U ? (d > c[i] ? int(d - c[i]) : 0) : U;
  }
  // the first row before gamma and beta, which are not waited for until its sums are there
  Unit<T> next[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) next[i].load((x + blockIdx.x * d) + c[i], left[i]);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
#pragma unroll
    for (int e = 0; e < U; ++e) g[i][e] = 1.f, b[i][e] = 0.f;
    if (gamma) load_floats(gamma + c[i], left[i], g[i]);
    if (beta) load_floats(beta + c[i], left[i], b[i]);
  }
  using Sums = BlockSums<MOST, 1>;
  __shared__ __align__(16) typename Sums::Row part;
  Sums::start(part);
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
    Unit<T> v[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = next[i];
    if (r + gridDim.x < rows)
#pragma unroll
      for (int i = 0; i < NV; ++i) next[i].load((x + (r + gridDim.x) * d) + c[i], left[i]);
    float s[1] = {0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < U; ++e) s[0] += v[i][e];
    Sums::sum(part, s, 0);
    const float m = s[0] / float(d);
    s[0] = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i].forget();
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < U; ++e) {
        const float w = v[i][e] - m;
        s[0] += e < left[i] ? w * w : 0.f;
      }
    Sums::sum(part, s, 1);
    const float rs = 1.f / sqrtf(s[0] / float(d) + eps);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      v[i].forget();
#pragma unroll
      for (int q = 0; q < U / 4; ++q) v[i].set(q, [&](int e) { return (v[i][e] - m) * rs * g[i][e] + b[i][e]; });
      v[i].store((y + r * d) + c[i], left[i]);
    }
    if (threadIdx.x == 0) {
      mean[r] = m;
      rstd[r] = rs;
    }
  }
}

// Rows of any length: three passes, of which the later ones find most rows in a cache (512 rows of 20000 fp32
// 24 us, their gradients 51; 500 of 1,000,001 bf16 1.1 and 1.7 ms).
constexpr int kLongThreads = 1024;

template <typename T>
__global__ __launch_bounds__(kLongThreads) void norm_long_kernel(const T *x, const float *gamma, const float *beta,
                                                                 int64_t rows, int64_t d, float eps, T *y, float *mean,
                                                                 float *rstd) {
  constexpr int U = kUnit<T>;
  using Sums = BlockSums<kLongThreads, 1>;
  __shared__ __align__(16) typename Sums::Row part;
  auto left = [&](int64_t c) { return d - c < U ? int(d - c) : U; };
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
    const T *xr = x + r * d;
    float s[1] = {0.f};
#pragma unroll 4
    for (int64_t c = threadIdx.x * U; c < d; c += kLongThreads * U) {
      Unit<T> v;
      v.load(xr + c, left(c));
#pragma unroll
      for (int e = 0; e < U; ++e) s[0] += v[e];
    }
    Sums::sum(part, s, 0);
    const float m = s[0] / float(d);
    s[0] = 0.f;
#pragma unroll 4
    for (int64_t c = threadIdx.x * U; c < d; c += kLongThreads * U) {
      const int n = left(c);
      Unit<T> v;
      v.load(xr + c, n);
#pragma unroll
      for (int e = 0; e < U; ++e) {
        const float w = v[e] - m;
        s[0] += e < n ? w * w : 0.f;
      }
    }
    Sums::sum(part, s, 1);
    const float rs = 1.f / sqrtf(s[0] / float(d) + eps);
#pragma unroll 2
    for (int64_t c = threadIdx.x * U; c < d; c += kLongThreads * U) {
      const int n = left(c);
      Unit<T> v;
      float g[U], b[U];
#pragma unroll
      for (int e = 0; e < U; ++e) g[e] = 1.f, b[e] = 0.f;
      v.load(xr + c, n);
      if (gamma) load_floats(gamma + c, n, g);
      if (beta) load_floats(beta + c, n, b);
#pragma unroll
      for (int q = 0; q < U / 4; ++q) v.set(q, [&](int e) { return (v[e] - m) * rs * g[e] + b[e]; });
      v.store((y + r * d) + c, n);
    }
    if (threadIdx.x == 0) {
      mean[r] = m;
      rstd[r] = rs;
    }
  }
}

// A block takes rows run * per .. of chunk i; sums[i][run][dgamma, dbeta][d], or the results themselves
// where a chunk is one run.
template <typename T, int MOST, int NV, bool DX>
__global__ __launch_bounds__(MOST) __attribute__((amdgpu_waves_per_eu(4))) void norm_grads_kernel(const T *x, const T *dy, const float *gamma, const float *mean,
                                                             const float *rstd, int N, int64_t n, int64_t d, int runs, int64_t per,
                                                             T *dx, float *sums, float *dgamma, float *dbeta) {
  constexpr int U = kUnit<T>;
  const uint32_t block = block_number();
  const int64_t i = block / runs, run = block % runs;
  if (i >= N) return;  // the whole block
  const int64_t r0 = i * n + run * per, r1 = run * per + per < n ? r0 + per : (i + 1) * n;
  const float inv = 1.f / float(d);
  // gamma in LDS, a thread's own: sixteen registers less let rows of 16384 bf16 be loaded a row ahead
  typedef float Quad __attribute__((ext_vector_type(4)));
  __shared__ Quad gs[NV * U / 4][MOST];
  float sg[NV][U], sb[NV][U];
  uint32_t c[NV];  // columns
  int left[NV];    // how many of a unit's there are
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    c[k] = (k * blockDim.x + threadIdx.x) * U;
    left[k] = d - c[k] < U ? (d > c[k] ? int(d - c[k]) : 0) : U;
    float g[U];
#pragma unroll
    for (int e = 0; e < U; ++e) g[e] = 1.f, sg[k][e] = sb[k][e] = 0.f;
    if (gamma && DX) load_floats(gamma + c[k], left[k], g);
#pragma unroll
    for (int q = 0; q < U / 4; ++q) gs[k * U / 4 + q][threadIdx.x] = Quad{g[4 * q], g[4 * q + 1], g[4 * q + 2], g[4 * q + 3]};
  }
  using Sums = BlockSums<MOST, 2>;
  __shared__ __align__(16) typename Sums::Row part;
  Sums::start(part);
  constexpr bool kAhead = NV <= 2;  // a row ahead, as far as registers go
  Unit<T> xn[NV], an[NV];
  float mn = 0.f, rn = 0.f;
  auto load = [&](int64_t r) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      xn[k].load((x + r * d) + c[k], left[k]);
      an[k].load((dy + r * d) + c[k], left[k]);
    }
    mn = mean[r];
    rn = rstd[r];
  };
  if (kAhead && r0 < r1) load(r0);
  for (int64_t r = r0; r < r1; ++r) {
    if (!kAhead) load(r);
    Unit<T> xr[NV], ar[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) xr[k] = xn[k], ar[k] = an[k];
    const float m = mn, rs = rn;
    if (kAhead && r + 1 < r1) load(r + 1);
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      xr[k].fill(left[k]);
      float ah = 0.f;
#pragma unroll
      for (int q = 0; q < U / 4; ++q) {
        const Quad g = gs[k * U / 4 + q][threadIdx.x];
#pragma unroll
        for (int j = 0; j < 4; ++j) {  // past the row dy is zero
          const int e = 4 * q + j;
          const float h = (xr[k][e] - m) * rs, v = ar[k][e], a = v * g[j];
          sg[k][e] += v * h;
          sb[k][e] += v;
          s[0] += a;
          ah += a * h;
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      s[1] += left[k] > 0 ? ah : 0.f;  // of a unit past the row h, of no value of it, may be infinite
    }
    if constexpr (!DX) continue;
    Sums::sum(part, s, int(r & 1));
    // rstd last: its square is past the largest float for rows of deviations below 2^-64 (eps = 0)
    const float ca = -(s[0] * inv), ch = -(s[1] * inv);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      xr[k].forget();
      ar[k].forget();
#pragma unroll
      for (int q = 0; q < U / 4; ++q) {
        const Quad g = gs[k * U / 4 + q][threadIdx.x];
        ar[k].set(q, [&](int e) { return rs * fmaf(ar[k][e], g[e % 4], fmaf((xr[k][e] - m) * rs, ch, ca)); });
        __builtin_amdgcn_sched_barrier(0);
      }
      ar[k].store((dx + r * d) + c[k], left[k]);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  float *og = runs > 1 ? sums + int64_t(block) * 2 * d : (dgamma ? dgamma + i * d : nullptr);
  float *ob = runs > 1 ? sums + (int64_t(block) * 2 + 1) * d : (dbeta ? dbeta + i * d : nullptr);
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    if (og && dgamma) store_floats(og + c[k], left[k], sg[k]);
    if (ob && dbeta) store_floats(ob + c[k], left[k], sb[k]);
  }
}

// dgamma, dbeta [N][d] from the runs' sums: COLUMNS per block, EACH threads a column
template <int COLUMNS, int EACH>
__global__ __launch_bounds__(COLUMNS *EACH) void norm_join_kernel(const float *sums, int64_t d, int runs, float *dgamma,
                                                                  float *dbeta) {
  __shared__ float part[EACH][COLUMNS];
  const int64_t groups = (d + COLUMNS - 1) / COLUMNS, which = blockIdx.x % 2;
  const int64_t i = blockIdx.x / 2 / groups, c = blockIdx.x / 2 % groups * COLUMNS + threadIdx.x % COLUMNS;
  const int g = threadIdx.x / COLUMNS;
  float *out = which ? dbeta : dgamma;
  if (!out) return;  // the whole block
  float s = 0.f;
  if (c < d) {
    const float *src = sums + (i * runs * 2 + which) * d + c;
#pragma unroll 8
    for (int run = g; run < runs; run += EACH) s += src[int64_t(run) * 2 * d];
  }
  if constexpr (EACH > 1) {
    part[g][threadIdx.x % COLUMNS] = s;
    __syncthreads();
    if (g > 0) return;
    s = 0.f;
#pragma unroll
    for (int k = 0; k < EACH; ++k) s += part[k][threadIdx.x];
  }
  if (c < d) out[i * d + c] = s;
}

// Rows of any length, a block per row.
template <typename T>
__global__ __launch_bounds__(kLongThreads) void norm_dx_long_kernel(const T *x, const T *dy, const float *gamma,
                                                                    const float *mean, const float *rstd, int64_t rows,
                                                                    int64_t d, T *dx) {
  constexpr int U = kUnit<T>;
  using Sums = BlockSums<kLongThreads, 2>;
  __shared__ __align__(16) typename Sums::Row part;
  auto left = [&](int64_t c) { return d - c < U ? int(d - c) : U; };
  int turn = 0;
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x, turn ^= 1) {
    const float m = mean[r], rs = rstd[r];
    float s[2] = {0.f, 0.f};
#pragma unroll 2
    for (int64_t c = threadIdx.x * U; c < d; c += kLongThreads * U) {
      const int n = left(c);
      Unit<T> v, a;
      float g[U];
#pragma unroll
      for (int e = 0; e < U; ++e) g[e] = 1.f;
      v.load((x + r * d) + c, n);
      a.load((dy + r * d) + c, n);
      v.fill(n);
      if (gamma) load_floats(gamma + c, n, g);
#pragma unroll
      for (int e = 0; e < U; ++e) {  // past the row dy is zero
        const float w = a[e] * g[e];
        s[0] += w;
        s[1] += w * ((v[e] - m) * rs);
      }
    }
    Sums::sum(part, s, turn);
    const float sa = s[0] / float(d), sah = s[1] / float(d);
#pragma unroll 2
    for (int64_t c = threadIdx.x * U; c < d; c += kLongThreads * U) {
      const int n = left(c);
      Unit<T> v, a;
      float g[U];
#pragma unroll
      for (int e = 0; e < U; ++e) g[e] = 1.f;
      v.load((x + r * d) + c, n);
      a.load((dy + r * d) + c, n);
      if (gamma) load_floats(gamma + c, n, g);
#pragma unroll
      for (int q = 0; q < U / 4; ++q)
        a.set(q, [&](int e) { return rs * (a[e] * g[e] - sa - (v[e] - m) * rs * sah); });
      a.store((dx + r * d) + c, n);
    }
  }
}

// A thread takes one unit's columns of a run of a chunk's rows; sums as of norm_grads_kernel.
template <typename T>
__global__ __launch_bounds__(kThreads) void norm_weights_long_kernel(const T *x, const T *dy, const float *mean,
                                                                     const float *rstd, int64_t n, int64_t d, int runs,
                                                                     int64_t per, float *sums, float *dgamma,
                                                                     float *dbeta) {
  constexpr int U = kUnit<T>;
  const int64_t groups = (d + kThreads * U - 1) / (kThreads * U), both = blockIdx.x / groups;
  const int64_t i = both / runs, run = both % runs, c = (blockIdx.x % groups * kThreads + threadIdx.x) * U;
  if (c >= d) return;
  const int left = d - c < U ? int(d - c) : U;
  const int64_t r0 = i * n + run * per, r1 = run * per + per < n ? r0 + per : (i + 1) * n;
  float g[U], b[U];
#pragma unroll
  for (int e = 0; e < U; ++e) g[e] = b[e] = 0.f;
#pragma unroll 4
  for (int64_t r = r0; r < r1; ++r) {
    Unit<T> v, a;
    v.load((x + r * d) + c, left);
    a.load((dy + r * d) + c, left);
    const float m = mean[r], rs = rstd[r];
#pragma unroll
    for (int e = 0; e < U; ++e) {
      g[e] += a[e] * ((v[e] - m) * rs);
      b[e] += a[e];
    }
  }
  if (dgamma) store_floats((runs > 1 ? sums + both * 2 * d : dgamma + i * d) + c, left, g);
  if (dbeta) store_floats((runs > 1 ? sums + (both * 2 + 1) * d : dbeta + i * d) + c, left, b);
}

// A row has as many threads as hold one or two of its 16-byte units each, eight values (two of fp32, one of
// bf16 up to 1024 threads: with two the gradients take 134 registers and more, 20 chunks of 500 x 4099
// 153 us, with one 106), four past 2048 units; past that it is not held.
constexpr int64_t kMostUnits = 4 * 1024;
template <typename T>
int units_each(int64_t units) {
  return units <= 64 || (sizeof(T) == 2 && units <= 1024) ? 1 : (units <= 2048 ? 2 : 4);
}
template <typename T>
int threads_for(int64_t units) {
  return int(ceil_div(ceil_div(units, units_each<T>(units)), kWave) * kWave);
}

// bf16 takes one, two or four units a thread, fp32 two or four but in the shortest rows
#define GCX_ROWS(threads, each, ...)           \
  if (each == 4) {                             \
    constexpr int MOST = 1024, NV = 4;         \
    __VA_ARGS__;                               \
  } else if (each == 1 && threads <= 64) {     \
    constexpr int MOST = 64, NV = 1;           \
    __VA_ARGS__;                               \
  } else if (threads > 512 || (each == 2 && sizeof(T) == 2)) { \
    if (each == 2) {                           \
      constexpr int MOST = 1024, NV = 2;       \
      __VA_ARGS__;                             \
    } else if constexpr (sizeof(T) == 2) {     \
      constexpr int MOST = 1024, NV = 1;       \
      __VA_ARGS__;                             \
    }                                          \
  } else if (threads > 256) {                  \
    constexpr int MOST = 512, NV = 8 / kUnit<T>; \
    __VA_ARGS__;                               \
  } else {                                     \
    constexpr int MOST = 256, NV = 8 / kUnit<T>; \
    __VA_ARGS__;                               \
  }

constexpr int kNormThreads = 2048;  // of a CU that blocks of norm_kernel are launched for, each taking row after row

template <typename T>
int launch_norm(const void *x, const float *gamma, const float *beta, int64_t rows, int64_t d, float eps, void *y,
                float *mean, float *rstd, hipStream_t st) {
  const T *xt = static_cast<const T *>(x);
  T *yt = static_cast<T *>(y);
  const int64_t units = ceil_div(d, kUnit<T>);
  if (units > kMostUnits) {
    hipLaunchKernelGGL(norm_long_kernel<T>, dim3(unsigned(std::min<int64_t>(rows, 1 << 16))), dim3(kLongThreads), 0, st, xt, gamma, beta, rows, d, eps, yt, mean, rstd);
    return launch_status();
  }
  const int threads = threads_for<T>(units), each = units_each<T>(units);
  const dim3 blocks(unsigned(std::min<int64_t>(rows, int64_t(cu_count()) * (kNormThreads / threads))));
  GCX_ROWS(threads, each, hipLaunchKernelGGL((norm_kernel<T, MOST, NV>), blocks, dim3(unsigned(threads)), 0, st, xt, gamma, beta, rows,
                                     d, eps, yt, mean, rstd))
  return launch_status();
}

// Runs of a chunk's rows, of eight rows or more: the least rounds of resident blocks (sixteen waves per CU or more)
// times what a block takes, its rows and about two more for what it loads first and leaves, and the join.
template <typename T>
int64_t runs_for(int64_t N, int64_t n, int64_t units) {
  if (units > kMostUnits)  // blocks of 256 units: eight to a CU, but eight rows or more each
    return std::max<int64_t>(1, std::min(n / 8, ceil_div(2048, N * ceil_div(units, kThreads))));
  const int waves = units_each<T>(units) == 1 ? 24 : 16;  // as registers allow
  const int64_t slots = 256 * std::max(1, waves * kWave / threads_for<T>(units)), most = std::max<int64_t>(1, std::min(n / 8, 2 * slots / N));
  int64_t best = 1, least = -1;
  for (int64_t runs = 1; runs <= most; runs += 1 + runs / 16) {
    const int64_t took = ceil_div(N * runs, slots) * (ceil_div(n, runs) + 2) + runs / 64;
    if (least < 0 || took < least) best = runs, least = took;
  }
  return best;
}

template <typename T>
int launch_grads(const void *x, const void *dy, const float *gamma, const float *mean, const float *rstd, int N, int n,
                 int64_t d, void *dx, float *dgamma, float *dbeta, float *sums, hipStream_t st) {
  const int64_t rows = int64_t(N) * n, units = ceil_div(d, kUnit<T>);
  const T *xt = static_cast<const T *>(x), *dyt = static_cast<const T *>(dy);
  T *dxt = static_cast<T *>(dx);
  const int64_t per = ceil_div(std::max(n, 1), runs_for<T>(N, n, units));
  const int runs = int(ceil_div(std::max(n, 1), per));
  if (units > kMostUnits) {
    if (dgamma || dbeta)
      hipLaunchKernelGGL(norm_weights_long_kernel<T>, dim3(unsigned(N * runs * ceil_div(units, kThreads))), dim3(kThreads), 0, st,
                         xt, dyt, mean, rstd, n, d, runs, per, sums, dgamma, dbeta);
    if (dx && rows > 0)
      hipLaunchKernelGGL(norm_dx_long_kernel<T>, dim3(unsigned(std::min<int64_t>(rows, 1 << 16))), dim3(kLongThreads), 0, st, xt,
                         dyt, gamma, mean, rstd, rows, d, dxt);
  } else {
    const int threads = threads_for<T>(units), each = units_each<T>(units);
    GCX_ROWS(threads, each, hipLaunchKernelGGL((dx ? norm_grads_kernel<T, MOST, NV, true> : norm_grads_kernel<T, MOST, NV, false>), blocks_of(int64_t(N) * runs),
                                     dim3(unsigned(threads)), 0, st, xt, dyt, gamma, mean, rstd, N, n, d, runs, per, dxt, sums, dgamma, dbeta))
  }
  if (runs > 1 && (dgamma || dbeta)) {
    auto join = [&](auto kernel, int columns, int threads) {
      hipLaunchKernelGGL(kernel, dim3(unsigned(2 * N * ceil_div(d, columns))), dim3(unsigned(threads)), 0, st, sums, d, runs,
                         dgamma, dbeta);
    };
    // threads a column: a chain of at most some tens of loads
    if (runs <= 8)
      join(norm_join_kernel<256, 1>, 256, 256);
    else if (runs <= 128)
      join(norm_join_kernel<64, 16>, 64, 1024);
    else
      join(norm_join_kernel<16, 64>, 16, 1024);
  }
  return launch_status();
}

}  // namespace
}  // namespace gcx

extern "C" int gc_layer_norm(const void *x, const float *gamma, const float *beta, int64_t rows, int64_t d, double eps,
                             int32_t dtype, void *y, float *mean, float *rstd, hipStream_t stream) {
  using namespace gcx;
  if (rows < 0 || d < 1 || !(eps >= 0.0) || (dtype != GC_F32 && dtype != GC_BF16)) return GC_EINVAL;
  if (!sizes_ok({rows, d})) return GC_EINVAL;
  if (rows == 0) return GC_OK;
  if (!x || !y || !mean || !rstd) return GC_EINVAL;
  const int dev = check_device();
  if (dev != GC_OK) return dev;
  (void)hipGetLastError();
  return dtype == GC_F32 ? launch_norm<float>(x, gamma, beta, rows, d, float(eps), y, mean, rstd, stream)
                         : launch_norm<__bf16>(x, gamma, beta, rows, d, float(eps), y, mean, rstd, stream);
}

extern "C" size_t gc_layer_norm_grads_workspace_size(int32_t N, int32_t n, int64_t d) {
  using namespace gcx;
  if (N < 1 || n < 1 || d < 1 || !sizes_ok({N, n, d}) || !sizes_ok({N, d})) return 0;
  const int64_t bf16 = ceil_div(d, kUnit<__bf16>), f32 = ceil_div(d, kUnit<float>);
  const int64_t runs = std::max(runs_for<__bf16>(N, n, bf16), runs_for<float>(N, n, f32));
  return runs > 1 ? size_t(N) * size_t(runs) * 8 * size_t(d) : 0;
}

extern "C" int gc_layer_norm_grads(const void *x, const void *dy, const float *gamma, const float *mean,
                                   const float *rstd, int32_t N, int32_t n, int64_t d, int32_t dtype, void *dx,
                                   float *dgamma, float *dbeta, void *workspace, size_t workspace_bytes,
                                   hipStream_t stream) {
  using namespace gcx;
  if (N < 0 || n < 0 || d < 1 || (dtype != GC_F32 && dtype != GC_BF16)) return GC_EINVAL;
  if (!sizes_ok({N, n, d}) || !sizes_ok({N, d}) || N * ceil_div(d, 16) > int64_t(1) << 29) return GC_EINVAL;
  if (N == 0) return GC_OK;
  if (n > 0 && (!x || !dy || !mean || !rstd)) return GC_EINVAL;
  if (!dx && !dgamma && !dbeta) return n > 0 ? GC_EINVAL : GC_OK;
  const size_t need = gc_layer_norm_grads_workspace_size(N, n, d);
  if (need && (!workspace || workspace_bytes < need || !aligned16(workspace))) return GC_EINVAL;
  const int dev = check_device();
  if (dev != GC_OK) return dev;
  (void)hipGetLastError();
  float *sums = static_cast<float *>(workspace);
  return dtype == GC_F32 ? launch_grads<float>(x, dy, gamma, mean, rstd, N, n, d, dx, dgamma, dbeta, sums, stream)
                         : launch_grads<__bf16>(x, dy, gamma, mean, rstd, N, n, d, dx, dgamma, dbeta, sums, stream);
}
