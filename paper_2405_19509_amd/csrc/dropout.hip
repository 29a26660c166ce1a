// Dropout whose mask is a counter-based generator's (gc_dropout).
#include "common.h"
#include "head.h"

namespace gcx {
namespace {

// Philox 4x32-10 (Salmon, Moraes, Dror, Shaw 2011): ten rounds of two 32 x 32 products.
__device__ __forceinline__ void philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1,
                                       uint32_t (&u)[4]) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = uint64_t(c0) * 0xD2511F53u, b = uint64_t(c2) * 0xCD9E8D57u;
    c0 = uint32_t(b >> 32) ^ c1 ^ k0;
    c1 = uint32_t(b);
    c2 = uint32_t(a >> 32) ^ c3 ^ k1;
    c3 = uint32_t(a);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  u[0] = c0;
  u[1] = c1;
  u[2] = c2;
  u[3] = c3;
}

// A thread takes one column group (4 Q columns, Q counters) of ROWS rows at a time, whose loads are under
// way together; TX threads lie along a row.  Vector loads need no alignment; a row's last group is taken
// apart where it is not whole.  Bound by memory (25,600 x 16384 bf16 with an addend 436 us, 5.8 TB/s), but for bf16
// without one: the generator's products keep the vector units busy all of its 335 to 369 us (a copy 323).
template <typename T, int Q, int ROWS>
__global__ __launch_bounds__(256) void dropout_kernel(const T *x, const T *addend, int64_t rows, int64_t d, int tx,
                                                      int64_t xblocks, uint64_t drop_below, float scale, uint32_t k0,
                                                      uint32_t k1, uint32_t step, int64_t row0, T *y) {
  constexpr int U = 4 * Q;
  typedef T Vec __attribute__((ext_vector_type(U), aligned(sizeof(T))));
  const int ty = 256 / tx, r_in = threadIdx.x / tx;
  const int64_t xb = blockIdx.x % xblocks, yb = blockIdx.x / xblocks, yblocks = gridDim.x / xblocks;
  const int64_t c = (xb * tx + threadIdx.x % tx) * U;
  if (c >= d) return;
  const bool whole = c + U <= d;
  for (int64_t r0 = yb * (ty * ROWS) + r_in; r0 < rows; r0 += yblocks * (ty * ROWS)) {
    Vec v[ROWS], a[ROWS];
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
      const int64_t r = r0 + k * ty;
      if (r >= rows) continue;
      const T *xs = x + r * d + c, *as = addend + r * d + c;
      if (whole) {
        v[k] = *reinterpret_cast<const Vec *>(xs);
        if (addend) a[k] = *reinterpret_cast<const Vec *>(as);
      } else {
#pragma unroll
        for (int e = 0; e < U; ++e)
          if (c + e < d) {
            v[k][e] = xs[e];
            if (addend) a[k][e] = as[e];
          }
      }
    }
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
      const int64_t r = r0 + k * ty;
      if (r >= rows) continue;
      const uint64_t row = uint64_t(row0) + uint64_t(r);
      Vec out;
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        uint32_t u[4];
        philox(uint32_t(c / 4 + q), step, uint32_t(row), uint32_t(row >> 32), k0, k1, u);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float w = u[e] >= drop_below ? to_f32(v[k][4 * q + e]) * scale : 0.f;
          out[4 * q + e] = from_f32<T>(addend ? to_f32(a[k][4 * q + e]) + w : w);
        }
      }
      T *dst = y + r * d + c;
      if (whole) {
        *reinterpret_cast<Vec *>(dst) = out;
      } else {
#pragma unroll
        for (int e = 0; e < U; ++e)
          if (c + e < d) dst[e] = out[e];
      }
    }
  }
}

template <typename T, int Q>
int launch_dropout(const void *x, const void *addend, int64_t rows, int64_t d, uint64_t below, float scale, uint64_t seed,
                   uint32_t step, int64_t row0, void *y, hipStream_t st) {
  constexpr int kRowsAtOnce = 2;
  const int64_t groups = ceil_div(d, 4 * Q);
  int tx = 1;
  while (tx < 256 && tx < groups) tx *= 2;
  const int64_t xblocks = ceil_div(groups, tx), per = int64_t(256 / tx) * kRowsAtOnce;
  const int64_t yblocks = std::max<int64_t>(1, std::min(ceil_div(rows, per), (int64_t(1) << 16) / xblocks));
  hipLaunchKernelGGL((dropout_kernel<T, Q, kRowsAtOnce>), dim3(unsigned(xblocks * yblocks)), dim3(256), 0, st,
                     static_cast<const T *>(x), static_cast<const T *>(addend), rows, d, tx, xblocks, below, scale,
                     uint32_t(seed), uint32_t(seed >> 32), step, row0, static_cast<T *>(y));
  return launch_status();
}

}  // namespace
}  // namespace gcx

extern "C" int gc_dropout(const void *x, const void *addend, int64_t rows, int64_t d, double p, uint64_t seed,
                          uint32_t step, int64_t row0, int32_t dtype, void *y, hipStream_t stream) {
  using namespace gcx;
  if (rows < 0 || d < 1 || row0 < 0 || !(p >= 0.0 && p <= 1.0)) return GC_EINVAL;
  if ((dtype != GC_F32 && dtype != GC_BF16) || !sizes_ok({rows, d}) || d > int64_t(1) << 32) return GC_EINVAL;
  if (rows == 0) return GC_OK;
  if (!x || !y) return GC_EINVAL;
  const int dev = check_device();
  if (dev != GC_OK) return dev;
  (void)hipGetLastError();
  const uint64_t below = uint64_t(p * 4294967296.0);
  const float scale = p < 1.0 ? float(1.0 / (1.0 - p)) : 0.f;
  return dtype == GC_F32 ? launch_dropout<float, 1>(x, addend, rows, d, below, scale, seed, step, row0, y, stream)
                         : launch_dropout<__bf16, 2>(x, addend, rows, d, below, scale, seed, step, row0, y, stream);
}
