// Softmax cross entropy over a vocabulary, in pieces of it, and its gradients per chunk.
//
// Three products (xent_mma.h), with a part of the logits at a time and never in memory:
//   z = H W^T          [rows][V]   reduced to a maximum and a sum per row and tile
//   dH = P W           [rows][d]   P of a piece of the vocabulary, from the logits made anew
//   G_i = P_i^T H_i    [V][d]
// bf16 enters the matrix cores as it is, with P rounded to bf16; what that leaves of a row's target, whose
// entry is nearly all of most rows' gradients, is added to dH and G in fp32 and as a second bf16 part (without:
// dH and G off by 2.4e-3, with 1.8e-3, of which 1.7e-3 is their own rounding to bf16).  fp32 enters
//   the logits and G as two fp16 parts of values scaled by a power of two (22 digits of every value down to
//     2^-18 of the largest that shares its scale, an error of 2^-40 of that one below), three products each:
//     H and W by row, P by column and chunk, from the largest of the chunk's rows (a kernel of its own), so
//     that rare entries of the vocabulary have gradients of their own size;
//   dH as three bf16 parts, six products: along a row of P there is no scale that the largest probability
//     and the smallest could share.
// The scales of H's rows are taken out of P before the sum over them, the others out of the result: exact.
// Few rows, or little work in all, take fp32 as it is, on the fp32 matrix instructions: what they lack in
// rate (a sixteenth of bf16's) is less than laying out W costs (see direct_pays).
// Infinities and NaN have no parts; a wave whose logits are not finite forms them again with the fp32
// matrix instructions, which treat them as the vector units do (5120 rows, V d = 8192 x 1024 with gradients 1470 us;
// with one entry at -infinity, so that every tile of it does, 3395).
#include <cfloat>
#include <cmath>

#include "common.h"
#include "head.h"
#include "xent_mma.h"

namespace gcx {
namespace {

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;

// 2^exponent <= |v| < 2 * 2^exponent, for normal v
__device__ __forceinline__ int exponent(float v) { return int(__float_as_uint(v) >> 23 & 255u) - 127; }
constexpr int kTop = 14;  // scaled values stay below 2^15, half of fp16's largest

// fp32 values from 3.396e38 on round past the largest bf16, kMostBf16.  The first of three parts is therefore that of
// kBelow times the value, which is at most kMostBf16; the other two hold the rest as well (1.5 * 2^-26 of it is left).
constexpr float kMostBf16 = 0x1.fep127f, kBelow = 0x1.fep-1f;

typedef __bf16 v4bf __attribute__((ext_vector_type(4)));
typedef _Float16 v4hf __attribute__((ext_vector_type(4)));

template <int NP>
using Part = std::conditional_t<NP == 0, float, std::conditional_t<NP == 2, _Float16, __bf16>>;

// ---------------------------------------------------------------------------------------
// operands laid out: rows of dp values (whole units of 16 bytes, zeros past d), rows without a target zero
// ---------------------------------------------------------------------------------------

// A wave per row.  NP = 0, 1: the values themselves; NP = 2: two planes of fp16 and the row's exponent exps[row]; NP = 3: three of bf16.
// clear: `count` words set to zero for a later kernel.
template <typename T, int NP>
__global__ __launch_bounds__(256) void lay_out_kernel(const T *src, int64_t rows, int64_t d, int64_t dp, const int32_t *label, int32_t V, Part<NP> *out, int *exps,
                                                      unsigned *clear, int64_t count) {
  typedef T Four __attribute__((ext_vector_type(4), aligned(sizeof(T))));  // rows start anywhere
  typedef Part<NP> Out __attribute__((ext_vector_type(4)));
  for (int64_t e = int64_t(block_number()) * 256 + threadIdx.x; e < count; e += int64_t(gridDim.x) * gridDim.y * 256) clear[e] = 0;
  const int lane = threadIdx.x % kWave;
  const int64_t r = int64_t(block_number()) * 4 + threadIdx.x / kWave;
  if (r >= rows) return;
  const T *row = src + r * d;
  bool zero = false;
  if (label) {
    const int32_t y = label[r];
    zero = y < 0 || y >= V;
  }
  auto four = [&](int64_t c) {
    v4f v = {0.f, 0.f, 0.f, 0.f};
    if (c + 4 <= d) {
      const Four u = *reinterpret_cast<const Four *>(row + c);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = to_f32(u[e]);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (c + e < d) v[e] = to_f32(row[c + e]);
    }
    return v;
  };
  int k = 0;
  if constexpr (NP == 2) {
    float top = 0.f;
    if (!zero)
      for (int64_t c = 4 * lane; c < d; c += 4 * kWave) {
        const v4f v = four(c);
#pragma unroll
        for (int e = 0; e < 4; ++e) top = fmaxf(top, fabsf(v[e]));
      }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, kWave));
    k = top > 0.f && top < INFINITY ? kTop - exponent(top) : 0;
    if (lane == 0) exps[r] = k;
  }
  for (int64_t c = 4 * lane; c < dp; c += 4 * kWave) {
    v4f v = {0.f, 0.f, 0.f, 0.f};
    if (!zero) v = four(c);
#pragma unroll
    for (int p = 0; p < (NP ? NP : 1); ++p) {
      Out w;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (NP == 2 && p == 0) v[e] = ldexpf(v[e], k);
        w[e] = static_cast<Part<NP>>(NP == 3 && p == 0 ? v[e] * kBelow : v[e]);
        v[e] -= static_cast<float>(w[e]);
      }
      *reinterpret_cast<Out *>(out + (p * rows + r) * dp + c) = w;
    }
  }
}

// ---------------------------------------------------------------------------------------
// logits
// ---------------------------------------------------------------------------------------

struct Matrix {  // rows of values of `size` bytes, in planes
  int size;
  const char *at;
  int64_t ld;     // bytes
  int64_t plane;  // bytes
  const int *exps;  // of its rows (two planes)
  // the operand of a block with k along the rows, from row r0 of `rows` on, from k0 on
  __device__ __forceinline__ Operand along(int64_t r0, int64_t rows, int64_t k0) const {
    return {at + r0 * ld + k0 * size, (rows - r0) * ld - k0 * size, plane, uint32_t(ld)};
  }
  // with k numbering the rows k0 .. k1 - 1, from column c0 on
  __device__ __forceinline__ Operand across(int64_t c0, int64_t k0, int64_t k1) const {
    return {at + k0 * ld + c0 * size, (k1 - k0) * ld - c0 * size, plane, uint32_t(ld)};
  }
};

struct Logits {  // a piece of the vocabulary: entries v0 .. v0 + width - 1
  Matrix W, H;   // W from entry v0 on
  int64_t rows, K;
  int64_t v0, width;
  const int32_t *label;
  const float *Wf, *Hf;  // two planes: the values themselves, rows of d
  int64_t d;
  Logits part(int64_t from, int64_t to) const {  // entries from .. to - 1 of it
    Logits p = *this;
    p.W.at += from * W.ld;
    if (W.exps) p.W.exps += from;
    if (Wf) p.Wf += from * d;
    p.v0 += from;
    p.width = to - from;
    return p;
  }
};

// The wave's logits: two planes' scales taken out, and those anew that are not finite.
template <class P>
__device__ __forceinline__ void unscale(const Logits &a, int64_t f0, int64_t s0, v16f (&acc)[P::FT][P::ST]) {
  if constexpr (P::NP == 2) {
    const int h = (threadIdx.x % kWave) >> 5, li = threadIdx.x & 31;
    bool bad = false;
#pragma unroll
    for (int f = 0; f < P::FT; ++f)
#pragma unroll
      for (int s = 0; s < P::ST; ++s)
#pragma unroll
        for (int i = 0; i < 16; ++i) bad = bad || !(fabsf(acc[f][s][i]) <= FLT_MAX);
#pragma unroll
    for (int s = 0; s < P::ST; ++s) {
      const int64_t t = s0 + 32 * s + li;
      const int kt = t < a.rows ? a.H.exps[t] : 0;
#pragma unroll
      for (int f = 0; f < P::FT; ++f)
#pragma unroll
        for (int g = 0; g < 4; ++g) {  // the exponents' memory goes on to a multiple of 256 entries
          const int4 kv = *reinterpret_cast<const int4 *>(a.W.exps + f0 + 32 * f + 8 * g + 4 * h);
          const int k[4] = {kv.x, kv.y, kv.z, kv.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[f][s][4 * g + e] = ldexpf(acc[f][s][4 * g + e], -kt - k[e]);
        }
    }
    if (__any(bad)) {
#pragma unroll 1
      for (int s = 0; s < P::ST; ++s) {
        const int64_t t = s0 + 32 * s + li;
        const float *y = a.Hf + (t < a.rows ? t : 0) * a.d;
#pragma unroll
        for (int f = 0; f < P::FT; ++f) {
          const int64_t v = f0 + 32 * f + li;
          const float *x = a.Wf + (v < a.width ? v : 0) * a.d;
          v16f z = {};
          for (int64_t k = 0; k < a.d; k += 2) {  // rows that do not exist repeat the first: not used
            const bool in = k + h < a.d;
            const float u = x[in ? k + h : 0], w = y[in ? k + h : 0];
            z = __builtin_amdgcn_mfma_f32_32x32x2f32(in ? u : 0.f, in ? w : 0.f, z, 0, 0, 0);
          }
#pragma unroll
          for (int j = 0; j < P::ST; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if (j == s && !(fabsf(acc[f][j][i]) <= FLT_MAX)) acc[f][j][i] = z[i];
        }
      }
    }
  }
}

// exp(v), v <= 0 a difference of logits.  The difference comes first: a logit times log2(e) is rounded to its own last
// digit, and past the largest float from 2.36e38 on.  (With one fma from that product instead: 4096 rows, V d = 131072 x
// 1024 bf16 forward 942 us to 930, 4600 rows, 32768 x 64 72.5 to 70.5.)
__device__ __forceinline__ float exp_of(float v) { return __builtin_amdgcn_exp2f(v * kLog2e); }

// The log-sum-exp less the target's logit from their largest logit on: exactly log(sum) where that is the target's,
// and never below 0.
__device__ __forceinline__ float loss_of(float largest, float sum, float target) {
  return (largest - target) + log2f(sum) * kLn2;
}

// The tile's share of each row, for the join, or the results themselves where one tile is all of the vocabulary
// (loss given): part[v tile][row] = (m, sum of exp(z - m)), m the largest of the tile's logits z; target[row] the target's
template <class P, int FB>
__global__ __launch_bounds__(P::Threads) void lse_part_kernel(Logits a, uint32_t nf, uint32_t ns, int64_t tile0, float2 *part,
                                                              float *target, int32_t V, float *loss, float *lse) {
  __shared__ __align__(1024) char lds[P::Lds];
  const int lane = threadIdx.x % kWave, li = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), wf = wave % P::WF, ws = wave / P::WF;
  float2 *red = reinterpret_cast<float2 *>(lds);               // [WF][TS]
  float *own = reinterpret_cast<float *>(red + P::WF * P::TS);  // [TS]: the targets' logits, where loss is given
  Pipe<P, true, true, FB> pipe(lds);
  int ft, st;
  if (!tile_of(block_number(), nf, ns, ft, st)) return;
  pipe.start(a.W.along(int64_t(ft) * P::TF, a.width, 0), a.H.along(int64_t(st) * P::TS, a.rows, 0), a.K);
  const int64_t f0 = int64_t(ft) * P::TF + wf * P::FT * 32, s0 = int64_t(st) * P::TS + ws * P::ST * 32;
  int32_t label[P::ST];
#pragma unroll
  for (int s = 0; s < P::ST; ++s) {
    const int64_t t = s0 + 32 * s + li;
    label[s] = t < a.rows ? a.label[t] : -1;
  }
  v16f acc[P::FT][P::ST];
  pipe.run(acc);
  unscale<P>(a, f0, s0, acc);
  const int inside = a.width - f0 < P::FT * 32 ? int(a.width - f0) : P::FT * 32;  // of the wave's entries
  if (inside < P::FT * 32) {
#pragma unroll
    for (int s = 0; s < P::ST; ++s)
#pragma unroll
      for (int f = 0; f < P::FT; ++f)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[f][s][i] = 32 * f + tile_f(i) < inside ? acc[f][s][i] : -INFINITY;
  }
#pragma unroll
  for (int s = 0; s < P::ST; ++s) {
    const int64_t v = label[s] >= 0 ? label[s] - a.v0 - f0 : -1;
    const int y = v >= 0 && v < P::FT * 32 ? int(v) : -1;
    if (__any(y >= 0)) {  // a target among the wave's entries
#pragma unroll
      for (int f = 0; f < P::FT; ++f)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (y == 32 * f + tile_f(i)) (loss ? own + (ws * P::ST + s) * 32 + li : target + s0 + 32 * s + li)[0] = acc[f][s][i];
    }
    float m = -INFINITY;
#pragma unroll
    for (int f = 0; f < P::FT; ++f)
#pragma unroll
      for (int i = 0; i < 16; ++i) m = fmaxf(m, acc[f][s][i]);
    m = fmaxf(m, __shfl_xor(m, 32, kWave));
    const float shift = m == -INFINITY ? 0.f : m;  // none but -inf: a sum of zeros
    // in four sums: what a long one that holds the largest's 1 rounds away of small terms is most of a small loss's error
    float four[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int f = 0; f < P::FT; ++f)
#pragma unroll
      for (int i = 0; i < 16; ++i) four[i % 4] += exp_of(acc[f][s][i] - shift);
    float sum = (four[0] + four[1]) + (four[2] + four[3]);
    sum += __shfl_xor(sum, 32, kWave);
    if (lane < 32) red[wf * P::TS + (ws * P::ST + s) * 32 + li] = make_float2(m, sum);
  }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  for (int c = threadIdx.x; c < P::TS; c += P::Threads) {
    const int64_t t = int64_t(st) * P::TS + c;
    if (t >= a.rows) continue;
    float m = -INFINITY, sum = 0.f;
#pragma unroll
    for (int w = 0; w < P::WF; ++w) m = fmaxf(m, red[w * P::TS + c].x);
    const float shift = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int w = 0; w < P::WF; ++w) sum += red[w * P::TS + c].y * exp_of(red[w * P::TS + c].x - shift);
    if (!loss) {
      part[(tile0 + ft) * a.rows + t] = make_float2(m, sum);
    } else {
      const int32_t y = a.label[t];
      lse[t] = shift + log2f(sum) * kLn2;
      loss[t] = y >= 0 && y < V ? loss_of(shift, sum, own[c]) : 0.f;
    }
  }
}

// kJoin rows per block, 256 / kJoin threads a row; sums in an order that the number of tiles fixes
constexpr int kJoin = 8;
__global__ __launch_bounds__(256) void lse_join_kernel(const float2 *part, const float *target, const int32_t *label,
                                                       int64_t rows, int32_t V, int64_t tiles, float *loss, float *lse) {
  constexpr int kEach = 256 / kJoin;
  __shared__ float2 red[kEach][kJoin];
  const int c = threadIdx.x % kJoin, g = threadIdx.x / kJoin;
  const int64_t r = int64_t(block_number()) * kJoin + c;
  float m = -INFINITY, sum = 0.f;
  if (r < rows) {
#pragma unroll 4
    for (int64_t p = g; p < tiles; p += kEach) {
      const float2 v = part[p * rows + r];
      const float top = fmaxf(m, v.x), shift = top == -INFINITY ? 0.f : top;
      sum = sum * exp_of(m - shift) + v.y * exp_of(v.x - shift);
      m = top;
    }
  }
  red[g][c] = make_float2(m, sum);
  __syncthreads();
  if (g > 0 || r >= rows) return;
  m = -INFINITY;
  for (int w = 0; w < kEach; ++w) m = fmaxf(m, red[w][c].x);
  const float shift = m == -INFINITY ? 0.f : m;
  float four[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int w = 0; w < kEach; ++w) four[w % 4] += red[w][c].y * exp_of(red[w][c].x - shift);
  sum = (four[0] + four[1]) + (four[2] + four[3]);
  lse[r] = shift + log2f(sum) * kLn2;
  const int32_t y = label[r];
  loss[r] = y >= 0 && y < V ? loss_of(shift, sum, target[r]) : 0.f;
}

// ---------------------------------------------------------------------------------------
// P of a piece
// ---------------------------------------------------------------------------------------

struct Probabilities {
  const float *lse, *dloss;
  int32_t V;
  int64_t ld, cols;  // values of a row of P, a multiple of 256; from the launch's first entry on
  __bf16 *P;   // bf16: [rows][ld]; two planes: for dH, in three planes; or NULL
  float *Q;    // fp32 as it is: P [rows][ld]; two planes: P over the scales of H's rows, for G; or NULL
  float *rest; // bf16: what rounding leaves of each row's target [rows]
};

// a finite value up to the largest bf16
__device__ __forceinline__ float within_bf16(float v) {
  return fabsf(v) < INFINITY ? __builtin_amdgcn_fmed3f(v, -kMostBf16, kMostBf16) : v;
}

template <class P, int FB>
__global__ __launch_bounds__(P::Threads) void p_kernel(Logits a, Probabilities b, uint32_t nf, uint32_t ns) {
  __shared__ __align__(1024) char lds[P::Lds];
  const int li = threadIdx.x & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), wf = wave % P::WF, ws = wave / P::WF;
  Pipe<P, true, true, FB> pipe(lds);
  int ft, st;
  if (!tile_of(block_number(), nf, ns, ft, st)) return;
  pipe.start(a.W.along(int64_t(ft) * P::TF, a.width, 0), a.H.along(int64_t(st) * P::TS, a.rows, 0), a.K);
  const int64_t f0 = int64_t(ft) * P::TF + wf * P::FT * 32, s0 = int64_t(st) * P::TS + ws * P::ST * 32;
  int32_t label[P::ST];
  float w[P::ST], lse[P::ST];
  int kh[P::ST];
#pragma unroll
  for (int s = 0; s < P::ST; ++s) {
    const int64_t t = s0 + 32 * s + li;
    const bool row = t < a.rows;
    label[s] = row ? a.label[t] : -1;
    w[s] = row && b.dloss ? b.dloss[t] : 1.f;
    lse[s] = row ? b.lse[t] : 0.f;
    kh[s] = P::NP == 2 && row ? a.H.exps[t] : 0;
  }
  v16f acc[P::FT][P::ST];
  pipe.run(acc);
  unscale<P>(a, f0, s0, acc);
  const int inside = a.width - f0 < P::FT * 32 ? int(a.width - f0) : P::FT * 32;  // of the wave's entries
#pragma unroll
  for (int s = 0; s < P::ST; ++s) {
    const bool there = label[s] >= 0 && label[s] < b.V;
    const float shift = there ? lse[s] : 0.f;
    const int64_t v = there ? label[s] - a.v0 - f0 : -1;
    const int y = v >= 0 && v < P::FT * 32 ? int(v) : -1;
#pragma unroll
    for (int f = 0; f < P::FT; ++f)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[f][s][i] = exp_of(acc[f][s][i] - shift);
    if (__any(y >= 0)) {
#pragma unroll
      for (int f = 0; f < P::FT; ++f)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[f][s][i] -= y == 32 * f + tile_f(i) ? 1.f : 0.f;
    }
#pragma unroll
    for (int f = 0; f < P::FT; ++f)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[f][s][i] = there ? acc[f][s][i] * w[s] : 0.f;
    if (inside < P::FT * 32) {
#pragma unroll
      for (int f = 0; f < P::FT; ++f)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[f][s][i] = 32 * f + tile_f(i) < inside ? acc[f][s][i] : 0.f;
    }
  }
  const int64_t rows = a.rows - s0, cols = b.cols - f0, to = s0 * b.ld + f0;
  if constexpr (P::NP == 1) {
#pragma unroll
    for (int s = 0; s < P::ST; ++s) {
      const int64_t v = label[s] >= 0 && label[s] < b.V ? label[s] - a.v0 - f0 : -1;
      const int y = v >= 0 && v < P::FT * 32 ? int(v) : -1;
      if (__any(y >= 0)) {
#pragma unroll
        for (int f = 0; f < P::FT; ++f)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (y == 32 * f + tile_f(i)) {
              const float v = acc[f][s][i];
              b.rest[s0 + 32 * s + li] = v - static_cast<float>(static_cast<__bf16>(within_bf16(v)));
            }
      }
      if (__any(fabsf(w[s]) > kMostBf16)) {  // so may P be
#pragma unroll
        for (int f = 0; f < P::FT; ++f)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[f][s][i] = within_bf16(acc[f][s][i]);
      }
    }
    store_tiles<P>(lds, b.P + to, b.ld, rows, cols, [&](int f, int s, int i) { return acc[f][s][i]; });
  } else {
    if (b.Q)
      store_tiles<P>(lds, b.Q + to, b.ld, rows, cols,
                     [&](int f, int s, int i) { return ldexpf(acc[f][s][i], -kh[s]); });
    if (b.P) {
#pragma unroll
      for (int p = 0; p < 3; ++p)
        store_tiles<P>(lds, b.P + p * a.rows * b.ld + to, b.ld, rows, cols, [&](int f, int s, int i) {  // leaves what the part leaves
          const float v = static_cast<float>(static_cast<__bf16>(p == 0 ? acc[f][s][i] * kBelow : acc[f][s][i]));
          acc[f][s][i] -= v;
          return v;
        });
    }
  }
}

// Q [rows][ld] as two fp16 planes, each column of a chunk scaled by its largest: first that, then the split.
// A block takes 64 columns of kColumnRows rows of a chunk, 16 threads of 4 along a row.
constexpr int kColumnRows = 128;

struct Columns {
  int64_t i, c, r0, r1;  // chunk, first of the thread's columns, rows of the chunk
  __device__ __forceinline__ Columns(int64_t n, int64_t ld) {
    const int64_t groups = ld / 64, runs = (n + kColumnRows - 1) / kColumnRows, g = blockIdx.x;
    i = g / groups / runs;
    c = g % groups * 64 + threadIdx.x % 16 * 4;
    r0 = g / groups % runs * kColumnRows;
    r1 = r0 + kColumnRows < n ? r0 + kColumnRows : n;
  }
};

// top[chunk][column]: the bits of the largest magnitude, which order as whole numbers; zero before
__global__ __launch_bounds__(256) void column_top_kernel(const float *Q, int64_t n, int64_t ld, unsigned *top) {
  __shared__ float red[16][64];
  const Columns b(n, ld);
  const int tc = threadIdx.x % 16, tr = threadIdx.x / 16;
  const float *src = Q + b.i * n * ld + b.c;
  v4f m = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int64_t r = b.r0 + tr; r < b.r1; r += 16) {
    const v4f v = *reinterpret_cast<const v4f *>(src + r * ld);
#pragma unroll
    for (int e = 0; e < 4; ++e) m[e] = fmaxf(m[e], fabsf(v[e]));
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) red[tr][4 * tc + e] = m[e];
  __syncthreads();
  if (threadIdx.x >= 64) return;
  float t = 0.f;
#pragma unroll
  for (int g = 0; g < 16; ++g) t = fmaxf(t, red[g][threadIdx.x]);
  atomicMax(top + b.i * ld + b.c - 4 * tc + threadIdx.x, __float_as_uint(t));
}

__device__ __forceinline__ int column_exponent(unsigned top) {
  const float m = __uint_as_float(top);
  return m > 0.f && m < INFINITY ? kTop - exponent(m) : 0;
}

__global__ __launch_bounds__(256) void split_columns_kernel(const float *Q, int64_t rows, int64_t n, int64_t ld,
                                                            const unsigned *top, _Float16 *out) {
  const Columns b(n, ld);
  const int tr = threadIdx.x / 16;
  int k[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) k[e] = column_exponent(top[b.i * ld + b.c + e]);
  const float *src = Q + b.i * n * ld + b.c;
  _Float16 *dst = out + b.i * n * ld + b.c;
#pragma unroll 4
  for (int64_t r = b.r0 + tr; r < b.r1; r += 16) {
    const v4f v = *reinterpret_cast<const v4f *>(src + r * ld);
    v4hf hi, lo;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float x = ldexpf(v[e], k[e]);
      hi[e] = static_cast<_Float16>(x);
      lo[e] = static_cast<_Float16>(x - static_cast<float>(hi[e]));
    }
    *reinterpret_cast<v4hf *>(dst + r * ld) = hi;
    *reinterpret_cast<v4hf *>(dst + rows * ld + r * ld) = lo;
  }
}

// ---------------------------------------------------------------------------------------
// dH and G
// ---------------------------------------------------------------------------------------

// large tiles of bf16 have no registers for the targets' rest
template <class P>
constexpr bool kDhAtOnce = P::NP != 1 || P::TF < 256;

// sum[split][row][dq] (+)= sum over the split's entries v of P[row][v] W[v], fp32; or dH itself where all of
// the vocabulary is one split
template <class P, typename T, int FB>
__global__ __launch_bounds__(P::Threads) void dh_kernel(Matrix Pm, Matrix W, int64_t rows, int64_t width, int64_t d, int64_t dq,
                                                        int64_t kper, bool first, uint32_t nf, uint32_t ns, uint32_t together, float *sum, T *dH,
                                                        const int32_t *label, int32_t V, const float *rest) {
  __shared__ __align__(1024) char lds[P::Lds];
  int ft, st;
  if (!tile_of(block_number(), nf, ns * together, ft, st)) return;
  const int64_t split = int64_t(blockIdx.z) * together + st / int(ns);
  st %= int(ns);
  const int lane = threadIdx.x % kWave, h = lane >> 5, li = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), wf = wave % P::WF, ws = wave / P::WF;
  const int64_t k0 = split * kper, k1 = k0 + kper < width ? k0 + kper : width;
  v16f acc[P::FT][P::ST];
  Pipe<P, false, true, FB> pipe(lds);
  pipe.start(W.across(int64_t(ft) * P::TF, k0, k1), Pm.along(int64_t(st) * P::TS, rows, k0), k1 - k0);
  pipe.run(acc);
  const int64_t f0 = int64_t(ft) * P::TF + wf * P::FT * 32, s0 = int64_t(st) * P::TS + ws * P::ST * 32;
  if (kDhAtOnce<P> && dH) {
    if constexpr (P::NP == 1) {
#pragma unroll
      for (int s = 0; s < P::ST; ++s) {
        const int64_t t = s0 + 32 * s + li;
        const int32_t y = t < rows ? label[t] : -1;
        if (y < 0 || y >= V) continue;
        const float r = rest[t];
        const char *w = W.at + y * W.ld;
#pragma unroll
        for (int f = 0; f < P::FT; ++f) {
#pragma unroll
          for (int g = 0; g < 4; ++g) {  // rows go on to whole units of 16 bytes
            const int64_t x = f0 + 32 * f + 8 * g + 4 * h;
            if (x >= d) continue;
            const v4bf v = *reinterpret_cast<const v4bf *>(w + x * 2);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[f][s][4 * g + e] += r * static_cast<float>(v[e]);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
    store_tiles<P>(lds, dH + s0 * d + f0, d, rows - s0, d - f0, [&](int f, int s, int i) { return acc[f][s][i]; });
    return;
  }
#pragma unroll
  for (int s = 0; s < P::ST; ++s) {
    const int64_t t = s0 + 32 * s + li;
    if (t >= rows) continue;
    float *dst = sum + (split * rows + t) * dq;
#pragma unroll
    for (int f = 0; f < P::FT; ++f)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int64_t x = f0 + 32 * f + 8 * g + 4 * h;
        if (x >= dq) continue;
        v4f v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = acc[f][s][4 * g + e];
        v4f *o = reinterpret_cast<v4f *>(dst + x);
        *o = first ? v : *o + v;
      }
  }
}

// dH[row][x] = the splits' sums, in an order that their number fixes, and for bf16 what rounding left of the
// target; 4 columns and every EACH'th split a thread
template <typename T, int EACH>
__global__ __launch_bounds__(256) void dh_finish_kernel(const float *sum, int64_t rows, int64_t d, int64_t dq, int splits,
                                                        const T *W, const int32_t *label, int32_t V, const float *rest,
                                                        T *dH) {
  constexpr int kHere = 256 / EACH;
  __shared__ v4f red[EACH > 1 ? EACH : 1][kHere];
  const int64_t quads = dq / 4;
  const int g = threadIdx.x / kHere, q = threadIdx.x % kHere;
  for (int64_t e0 = int64_t(blockIdx.x) * kHere; e0 < rows * quads; e0 += int64_t(gridDim.x) * kHere) {
    const int64_t e = e0 + q, r = e / quads, x = e % quads * 4;
    const bool in = e < rows * quads;
    v4f v = {0.f, 0.f, 0.f, 0.f};
    if (in) {
#pragma unroll 8
      for (int s = g; s < splits; s += EACH) v += *reinterpret_cast<const v4f *>(sum + (s * rows + r) * dq + x);
    }
    if constexpr (EACH > 1) {
      __syncthreads();  // what the round before left has been read
      red[g][q] = v;
      __syncthreads();
      if (g > 0) continue;
#pragma unroll
      for (int k = 1; k < EACH; ++k) v += red[k][q];
    }
    if (!in) continue;
    if constexpr (sizeof(T) == 2) {
      const int32_t y = label[r];
      if (y >= 0 && y < V)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (x + j < d) v[j] += rest[r] * to_f32(W[y * d + x + j]);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (x + j < d) dH[r * d + x + j] = from_f32<T>(v[j]);
  }
}

// Adds to the block's tile of G what rounding left of its targets: of the chunk's tokens those whose target is
// among the tile's TS entries are listed, and each 64 of them are one more stage, their rows of H against a
// matrix that has one value a token.  labels: the thread's of the first kAhead rounds of the chunk's tokens.
constexpr int kAhead = 4;
template <class P>
__device__ void add_rest(char *lds, const int32_t (&labels)[kAhead], const int32_t *label, const float *rest, const Matrix &H,
                         int64_t n, int64_t dp, int64_t v0, int entries, int64_t x0, v16f (&acc)[P::FT][P::ST]) {
  using FL = Loader<P, P::TF, false>;
  using SL = Loader<P, P::TS, false>;
  constexpr int kMost = 2 * P::Threads, kStage = 64;  // tokens listed, and taken at a time
  static_assert(P::Stage + kMost * 8 + 256 <= P::Lds && P::BK == kStage, "fits");
  int2 *list = reinterpret_cast<int2 *>(lds + P::Stage);
  int *counts = reinterpret_cast<int *>(list + kMost);
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int wf = wave % P::WF, ws = wave / P::WF;
  int listed = 0;
  auto take = [&](int first, int count) {
    for (int e = tid; e < kStage * (P::TF / 8); e += P::Threads) {
      const int k = e / (P::TF / 8), u = e % (P::TF / 8);
      uint4 v = make_uint4(0, 0, 0, 0);
      if (k < count && x0 + 8 * u < dp) v = *reinterpret_cast<const uint4 *>(H.at + list[first + k].x * H.ld + (x0 + 8 * u) * 2);
      *reinterpret_cast<uint4 *>(lds + k * (P::TF * 2) + (u ^ FL::swizzle(k)) * 16) = v;
    }
    char *sl = lds + P::TF * P::Row;
    for (int e = tid; e < kStage * (P::TS / 8); e += P::Threads) reinterpret_cast<uint4 *>(sl)[e] = make_uint4(0, 0, 0, 0);
    __syncthreads();
    if (tid < count) {
      const int2 it = list[first + tid];
      *reinterpret_cast<__bf16 *>(sl + tid * (P::TS * 2) + ((it.y >> 3) ^ SL::swizzle(tid)) * 16 + (it.y & 7) * 2) =
          static_cast<__bf16>(rest[it.x]);
    }
    __syncthreads();
    for (int kk = 0; kk * 16 < count; ++kk) {
      typename P::Frag f[P::FT], s[P::ST];
#pragma unroll
      for (int i = 0; i < P::ST; ++i) s[i] = fragment<P, P::TS, false>(sl, 0, (ws * P::ST + i) * 32, kk);
#pragma unroll
      for (int i = 0; i < P::FT; ++i) f[i] = fragment<P, P::TF, false>(lds, 0, (wf * P::FT + i) * 32, kk);
#pragma unroll
      for (int i = 0; i < P::FT; ++i)
#pragma unroll
        for (int j = 0; j < P::ST; ++j) acc[i][j] = mfma32(f[i], s[j], acc[i][j]);
    }
    __syncthreads();
  };
  for (int64_t t0 = 0, round = 0; t0 < n; t0 += P::Threads, ++round) {
    const int64_t t = t0 + tid;
    int32_t y = round == 0 ? labels[0] : (round == 1 ? labels[1] : (round == 2 ? labels[2] : labels[3]));
    if (round >= kAhead) y = t < n ? label[t] : -1;
    const int64_t c = int64_t(y) - v0;
    const bool hit = y >= 0 && c >= 0 && c < entries;
    const unsigned long long hits = __ballot(hit);
    if (lane == 0) counts[wave] = __popcll(hits);
    __syncthreads();
    int at = listed, all = 0;
    for (int w = 0; w < P::Waves; ++w) {
      at += w < wave ? counts[w] : 0;
      all += counts[w];
    }
    if (hit) list[at + __popcll(hits & ((1ull << lane) - 1))] = make_int2(int(t), int(c));
    listed += all;
    __syncthreads();
    if (listed > kMost - P::Threads || t0 + P::Threads >= n) {  // no room for another round, or the last
      for (int k = 0; k < listed; k += kStage) take(k, listed - k < kStage ? listed - k : kStage);
      listed = 0;
    }
  }
}

// G[i][v0 + v][x] = sum over the rows t of chunk i of P[t][v] H[t][x]
template <class P, typename T>
__global__ __launch_bounds__(P::Threads) void g_kernel(Matrix Pm, Matrix H, int64_t n, int64_t width, int64_t ld, int64_t d,
                                                       int64_t dp, int64_t V, int64_t v0, uint32_t nf, uint32_t ns, uint32_t N,
                                                       const unsigned *top, const int32_t *label, const float *rest, T *G) {
  __shared__ __align__(1024) char lds[P::Lds];
  const int li = threadIdx.x & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), wf = wave % P::WF, ws = wave / P::WF;
  Pipe<P, false, false> pipe(lds);
  int ft, st;
  if (!tile_of(block_number(), nf, ns * N, ft, st)) return;
  const int64_t i = st / int(ns), c = st % int(ns);
  pipe.start(H.across(int64_t(ft) * P::TF, i * n, (i + 1) * n), Pm.across(c * P::TS, i * n, (i + 1) * n), n);
  const int64_t f0 = int64_t(ft) * P::TF + wf * P::FT * 32, s0 = c * P::TS + ws * P::ST * 32;
  int k[P::ST];
#pragma unroll
  for (int s = 0; s < P::ST; ++s) {
    const int64_t v = s0 + 32 * s + li;
    k[s] = P::NP == 2 && v < ld ? -column_exponent(top[i * ld + v]) : 0;
  }
  int32_t labels[kAhead];
  if constexpr (P::NP == 1)
#pragma unroll
    for (int q = 0; q < kAhead; ++q) labels[q] = q * P::Threads + threadIdx.x < n ? label[i * n + q * P::Threads + threadIdx.x] : -1;
  v16f acc[P::FT][P::ST];
  pipe.run(acc);
  if constexpr (P::NP == 1) {
    const int entries = width - c * P::TS < P::TS ? int(width - c * P::TS) : P::TS;
    Matrix Hi = H;
    Hi.at += i * n * H.ld;
    add_rest<P>(lds, labels, label + i * n, rest + i * n, Hi, n, dp, v0 + c * P::TS, entries, int64_t(ft) * P::TF, acc);
  }
  store_tiles<P>(lds, G + (i * V + v0 + s0) * d + f0, d, width - s0, d - f0, [&](int f, int s, int j) {
    return P::NP == 2 ? ldexpf(acc[f][s][j], k[s]) : acc[f][s][j];
  });
}

// The same for chunks of few tokens, whose G is all stores: a thread holds 16 bytes' columns of the chunk's rows of
// H, at most MOST, and forms theirs for one entry of the vocabulary after another, P of kFewEntries entries in LDS.
constexpr int kFewEntries = 512;
template <int NP, typename T, int MOST>
__global__ __launch_bounds__(256) void g_few_kernel(const char *Pm, int64_t ld, const char *H, int64_t dp, int64_t rows, int n,
                                                    int64_t width, int64_t d, int64_t V, int64_t v0, int tx, uint32_t nx,
                                                    uint32_t nv, int entries, const int32_t *label, const float *rest, T *G) {
  constexpr int U = 16 / sizeof(T);
  typedef Part<NP> Row __attribute__((ext_vector_type(U)));
  typedef T Unit __attribute__((ext_vector_type(U)));
  typedef uint32_t Words __attribute__((ext_vector_type(4)));
  typedef uint32_t Anywhere __attribute__((ext_vector_type(4), aligned(2)));
  __shared__ __align__(16) float p[kFewEntries][MOST + (MOST > 4 ? 4 : 0)];  // neighbours' writes to other banks
  const uint32_t block = block_number();
  const int64_t i = block / nx / nv, first = int64_t(block / nx % nv) * entries;
  if (i * n >= rows) return;  // the whole block
  const int64_t x = (int64_t(block % nx) * tx + threadIdx.x % tx) * U;
  const int here = width - first < entries ? int(width - first) : entries;
  for (int e = threadIdx.x; e < MOST * entries; e += 256) {
    const int t = e / entries, v = e % entries;
    float w = 0.f;
    if (t < n && v < here) {
      const int64_t at = (i * n + t) * ld + first + v;
      if constexpr (NP == 1) {
        w = static_cast<float>(reinterpret_cast<const __bf16 *>(Pm)[at]);
        if (label[i * n + t] == v0 + first + v) w += rest[i * n + t];
      } else {
        w = reinterpret_cast<const float *>(Pm)[at];
      }
    }
    p[v][t] = w;
  }
  float h[MOST][U];
#pragma unroll
  for (int t = 0; t < MOST; ++t)
#pragma unroll
    for (int e = 0; e < U; ++e) h[t][e] = 0.f;
  if (x < d) {
#pragma unroll
    for (int t = 0; t < MOST; ++t)
      if (t < n)
#pragma unroll
        for (int plane = 0; plane < (NP ? NP : 1); ++plane) {  // rows go on to whole units; two planes: P is over their scale
          const Row v = *reinterpret_cast<const Row *>(reinterpret_cast<const Part<NP> *>(H) + (plane * rows + i * n + t) * dp + x);
#pragma unroll
          for (int e = 0; e < U; ++e) h[t][e] += static_cast<float>(v[e]);
        }
  }
  __syncthreads();
  if (x >= d) return;
  T *dst = G + (i * V + v0 + first) * d + x;
  for (int v = threadIdx.x / tx; v < here; v += 256 / tx) {
    float s[U];
#pragma unroll
    for (int e = 0; e < U; ++e) s[e] = 0.f;
#pragma unroll
    for (int t = 0; t < MOST; ++t) {
      const float w = p[v][t];
#pragma unroll
      for (int e = 0; e < U; ++e) s[e] = fmaf(w, h[t][e], s[e]);
    }
    Unit out;
#pragma unroll
    for (int e = 0; e < U; ++e) out[e] = from_f32<T>(s[e]);
    if (x + U <= d) {
      *reinterpret_cast<Anywhere *>(dst + v * d) = __builtin_bit_cast(Words, out);
    } else {
#pragma unroll
      for (int e = 0; e < U; ++e)
        if (x + e < d) dst[v * d + e] = out[e];
    }
  }
}

template <typename T>
__global__ __launch_bounds__(256) void zero_kernel(T *out, int64_t count) {
  for (int64_t e = int64_t(blockIdx.x) * 256 + threadIdx.x; e < count; e += int64_t(gridDim.x) * 256) out[e] = from_f32<T>(0.f);
}

// ---------------------------------------------------------------------------------------
// plans
// ---------------------------------------------------------------------------------------

constexpr int kPad = 256;  // the largest tile: pieces are multiples of it
// Tokens per chunk up to which G is formed by the vector units (us, with P, against the matrix cores: fp32 2 chunks
// of 4, V d = 65536 x 216, 41 / 62; 9 of 8, 79019 x 117, 126 / 173; 1 of 12, 65536 x 4096, 612 / 695; 10 of 16, 10007 x
// 1001, 168 / 198; 16 of 16, 8192 x 1024, 184 / 175; bf16 the first two 26 / 38 and 83 / 103, the last two 100 / 92
// and 89 / 84): in fp32 the lines cross about 16 tokens, in bf16 between 8 and 16.
template <typename T>
constexpr int kFewRows = sizeof(T) == 4 ? 16 : 8;
constexpr int64_t kMaxSplits = 512;

constexpr int stage_k(int NP) { return NP == 1 ? 64 : (NP == 3 ? 16 : 32); }
template <int NP>
using Large = Shape<NP, 256, 256, 2, 4, 2, stage_k(NP)>;
template <int NP>
using Middle = Shape<NP, 128, 128, 2, 2, 2, stage_k(NP)>;
template <int NP>
using Narrow = Shape<NP, 128, 32, 4, 1, 4, stage_k(NP)>;

int64_t up(int64_t v, int64_t to) { return ceil_div(v, to) * to; }

enum Size { kLarge, kMiddle, kNarrow };

int64_t tiles(Size z, int64_t f, int64_t s, int64_t batch, int64_t &nf, int64_t &ns) {
  nf = ceil_div(f, z == kLarge ? 256 : 128);
  ns = ceil_div(s, z == kLarge ? 256 : (z == kMiddle ? 128 : 32));
  return nf * ns * batch;
}

// What a product takes in us, about: rounds of the blocks that are resident at once (one large tile per CU,
// one or two of the others), each a time per 1024 k and one for the rest.  Measured for bf16: 64 to 4096 rows,
// V d of 100 x 64 to 32768 x 4096, every size of tile; `products` matrix instructions for each of bf16's.
float cost(Size z, int64_t total, int64_t K, float products) {
  const float a[3] = {27.f, 18.f, 8.3f}, alone[3] = {27.f, 12.5f, 6.6f}, rest[3] = {6.f, 4.f, 2.5f};
  const bool few = total <= 256;
  const float rounds = few ? 1.f : float(ceil_div(total, z == kLarge ? 256 : 512));
  return rounds * (products * (few ? alone[z] : a[z]) * float(K) / 1024.f + rest[z]);
}

// matrix instructions per k against bf16's; fp32 as it is has a sixteenth of the rate, but a narrow tile's
// time is not all in them (15 us for 1024 k alone)
constexpr float products_of(int NP) { return NP == 1 ? 1.f : (NP == 2 ? 3.f : (NP == 3 ? 6.f : 2.5f)); }

Size size_for(int64_t f, int64_t s, int64_t batch, int64_t K, int NP) {
  int64_t nf, ns;
  Size best = kNarrow;
  float least = cost(kNarrow, tiles(kNarrow, f, s, batch, nf, ns), K, products_of(NP));
  for (Size z : {kMiddle, kLarge}) {
    if (NP == 0 && z == kLarge) continue;
    const float c = cost(z, tiles(z, f, s, batch, nf, ns), K, NP == 0 ? 5.f : products_of(NP));
    if (c < least) best = z, least = c;
  }
  return best;
}

// The logits' tiles of w entries: large ones in whole rounds of the CUs and the rest in the size that suits it, where that
// is less by a twentieth than one size for all (1000 rows, V d = 50000 x 1000 fp32 forward 472 us, so 427; 2000 rows, 10240 x
// 2048 bf16 99 and 94).
struct Tiling {
  int64_t first;  // entries of `size`; the rest of `then`
  Size size, then;
};
Tiling tiling(int64_t w, int64_t rows, int64_t K, int NP) {
  int64_t nf, ns;
  Tiling t{w, size_for(w, rows, 1, K, NP), kNarrow};
  if (NP == 0) return t;
  const float products = products_of(NP);
  const int64_t all = tiles(kLarge, w, rows, 1, nf, ns), first = all / 256 * 256 / ns * 256;
  if (first <= 0 || first >= w || all > 4096) return t;
  const Size then = size_for(w - first, rows, 1, K, NP);
  const float both = cost(kLarge, tiles(kLarge, first, rows, 1, nf, ns), K, products) +
                     cost(then, tiles(then, w - first, rows, 1, nf, ns), K, products);
  return both * 1.05f < cost(t.size, tiles(t.size, w, rows, 1, nf, ns), K, products) ? Tiling{first, kLarge, then} : t;
}

// fp32: laying out W for the 16-bit matrix cores (twice for a gradient) reads and writes it some times over,
// which few rows do not pay for (us, forward and gradients, as it is / laid out: 160 rows, V d = 32768 x 4096
// 1665 / 1838, 24810 x 484 219 / 273; 200 rows 2236 / 1942 and 292 / 246; 200 rows, 8192 x 1000 176 / 201)
bool direct_pays(int64_t rows, int64_t V, int64_t d) { return rows <= 160 || rows * V * d <= int64_t(1) << 27; }

dim3 grid(int64_t total) { return blocks_of(up(total, 8)); }

// One workspace, cut into pieces of whole 256 bytes; with base NULL only the size.
struct Cut {
  char *base;
  size_t used = 0;
  template <typename T>
  T *take(int64_t count) {
    T *p = base ? reinterpret_cast<T *>(base + used) : nullptr;
    used += size_t(up(count * int64_t(sizeof(T)), 256));
    return p;
  }
};

struct Plan {
  int64_t rows, N, n, V, d, dp, dq, width, ld;
  int NP;
  // workspace
  char *H, *W, *W3;
  int *hexps, *wexps;
  unsigned *top;
  float2 *part;
  float *target, *sum, *Q, *rest;
  char *P, *P2;
  Size dh_size;
  int64_t splits, kper;
  size_t bytes;
};

// entries of the vocabulary per piece: P and the piece's W of up to 2^26 values
int64_t piece(int64_t rows, int64_t V, int64_t dp) {
  return std::min(up(V, kPad), std::max<int64_t>(kPad, (int64_t(1) << 26) / std::max(rows, dp) / kPad * kPad));
}

Plan plan(int64_t N, int64_t n, int64_t V, int64_t d, int32_t dtype, bool grads, void *ws) {
  Plan p{};
  p.N = N;
  p.n = n;
  p.rows = N * n;
  p.V = V;
  p.d = d;
  p.dq = up(d, 4);
  p.NP = dtype == GC_BF16 ? 1 : (direct_pays(p.rows, V, d) ? 0 : 2);
  p.dp = up(d, p.NP == 0 ? 4 : 8);  // whole units of 16 bytes: d itself where rows are taken as they are
  p.width = piece(p.rows, V, p.dp);
  p.ld = p.width;
  Cut c{static_cast<char *>(ws)};
  const int64_t bytes = p.NP == 1 ? 2 : 4;  // of a value, laid out
  p.H = c.take<char>(bytes * p.rows * p.dp);
  if (p.NP > 0) p.W = c.take<char>(bytes * p.width * p.dp);
  if (p.NP == 2) {
    p.hexps = c.take<int>(p.rows);
    p.wexps = c.take<int>(p.width);
  }
  if (!grads) {
    p.part = c.take<float2>(p.rows * ceil_div(V, 128));
    p.target = c.take<float>(p.rows);
  } else {
    if (p.NP == 1) p.rest = c.take<float>(p.rows);
    if (p.NP > 0) p.P = c.take<char>(2 * (p.NP == 2 ? 3 : 1) * p.rows * p.ld);
    if (p.NP != 1) p.Q = c.take<float>(p.rows * p.ld);
    if (p.NP == 2) {
      p.W3 = c.take<char>(6 * p.width * p.dp);
      p.P2 = c.take<char>(4 * p.rows * p.ld);
      p.top = c.take<unsigned>(N * p.ld);
    }
    // the piece's entries split over blocks, whose sums are written, read and joined
    const int64_t w = std::min(p.width, V);
    float least = 0.f;
    for (int64_t splits = 1; splits <= kMaxSplits && splits <= ceil_div(w, 128); splits += std::max<int64_t>(1, splits / 8)) {
      const int64_t kper = up(ceil_div(w, splits), 64);
      if (ceil_div(w, kper) != splits) continue;
      const int NP = p.NP == 2 ? 3 : p.NP;
      const Size z = size_for(d, p.rows, splits, kper, NP);
      int64_t nf, ns;
      const float us = cost(z, tiles(z, d, p.rows, splits, nf, ns), kper, z == kNarrow || NP ? products_of(NP) : 5.f) +
                       (splits > 1 || w < V ? 2.5f : 0.f) + float(splits * p.rows * p.dq) * (8.f / 4e6f);
      if (splits == 1 || us < least) {
        least = us;
        p.splits = splits;
        p.kper = kper;
        p.dh_size = z;
      }
    }
    p.sum = c.take<float>(p.splits * p.rows * p.dq);
  }
  p.bytes = c.used;
  return p;
}

// Tiles are numbered in 32 bits.  The kernels over P's columns take one row of the grid, past which P does not fit a
// device.
bool xent_sizes_ok(int64_t rows, int64_t N, int64_t V, int64_t d, int32_t dtype) {
  return rows >= 0 && N >= 0 && V >= 1 && d >= 1 && d <= int64_t(1) << 20 && (dtype == GC_F32 || dtype == GC_BF16) &&
         rows <= int64_t(1) << 31 && sizes_ok({rows, d}) && sizes_ok({rows, V}) && sizes_ok({N, V, d}) &&
         // the smallest tiles
         sizes_ok({ceil_div(rows, 32), ceil_div(V, 128)}) && ceil_div(rows, 32) * ceil_div(V, 128) < int64_t(1) << 30 &&
         ceil_div(rows, 32) * ceil_div(d, 128) < int64_t(1) << 30 &&
         N * ceil_div(d, 128) * ceil_div(std::min(V, piece(rows, V, up(d, 8))), 32) < int64_t(1) << 30 &&
         (dtype == GC_BF16 || direct_pays(rows, V, d) || rows <= kFewRows<float> * N ||
          grid_ok(N * (piece(rows, V, up(d, 8)) / 64) * ceil_div(rows / N, kColumnRows), 256));
}

#define GCX_SHAPE(size, NP, ...)           \
  switch (size) {                          \
    case kLarge: {                         \
      if constexpr (NP > 0) {              \
        using P = Large<NP>;               \
        __VA_ARGS__;                       \
      }                                    \
      break;                               \
    }                                      \
    case kMiddle: {                        \
      using P = Middle<NP>;                \
      __VA_ARGS__;                         \
      break;                               \
    }                                      \
    default: {                             \
      using P = Narrow<NP>;                \
      __VA_ARGS__;                         \
    }                                      \
  }

template <typename T, int NP>
void lay_out(const void *src, int64_t first, int64_t rows, int64_t d, int64_t dp, const int32_t *label, int32_t V, void *out,
             int *exps, hipStream_t st, unsigned *clear = nullptr, int64_t count = 0) {
  const T *s = static_cast<const T *>(src) + first * d;
  hipLaunchKernelGGL((lay_out_kernel<T, NP>), blocks_of(ceil_div(rows, 4)), dim3(256), 0, st, s, rows, d, dp,
                     label, V, static_cast<Part<NP> *>(out), exps, clear, count);
}

// The kernels take rows as they are where those start on 16 bytes and hold whole units of them.
template <typename T>
bool as_is(const void *p, int64_t d) {
  return d * int64_t(sizeof(T)) % 16 == 0 && aligned16(p);
}

// W's rows off 16 bytes: fp32 as it is loads them by single values (us, forward and gradients, against a copy of W in whole
// units: 32 rows, V d = 32768 x 3843 136 / 424 and 502 / 697, 18605 x 2022 69 / 112 and 155 / 200; 1000 x 3001, few tiles, 93 / 86
// and 115 / 107).
template <int NP, typename T, class F>
void by_alignment(const void *W, int64_t d, F f) {
  if constexpr (NP == 0) {
    if (!as_is<T>(W, d)) return f(std::integral_constant<int, 4>());
  }
  f(std::integral_constant<int, 16>());
}

// The piece's rows of W: where they are, or laid out anew.
template <typename T, int NP>
Matrix weights(const Plan &p, const void *W, int64_t v0, int64_t w, hipStream_t st) {
  constexpr int size = NP ? 2 : 4;
  if (NP == 0 || (NP == 1 && as_is<T>(W, p.d))) return {size, static_cast<const char *>(W) + v0 * p.d * size, p.d * size, 0, nullptr};
  lay_out<T, NP>(W, v0, w, p.d, p.dp, nullptr, 0, p.W, p.wexps, st, p.top, p.top ? p.N * p.ld : 0);
  return {size, p.W, p.dp * size, w * p.dp * size, p.wexps};
}

template <typename T, int NP>
int launch_xent(const Plan &p, const void *H, const void *W, const int32_t *label, float *loss, float *lse, hipStream_t st) {
  constexpr int bytes = NP ? 2 : 4;
  Matrix Hm{bytes, static_cast<const char *>(H), p.d * bytes, 0, nullptr};
  if (NP == 2 || !as_is<T>(H, p.d)) {
    lay_out<T, NP>(H, 0, p.rows, p.d, p.dp, nullptr, 0, p.H, p.hexps, st);
    Hm = {bytes, p.H, p.dp * bytes, p.rows * p.dp * bytes, p.hexps};
  }
  // W as it is needs no pieces
  const int64_t width = NP == 0 || (NP == 1 && as_is<T>(W, p.d)) ? up(p.V, kPad) : p.width;
  int64_t nf, ns, tile0 = 0;
  const bool at_once = p.V <= (size_for(p.V, p.rows, 1, p.d, NP) == kLarge ? 256 : 128);  // one tile of the vocabulary
  for (int64_t v0 = 0; v0 < p.V; v0 += width) {
    const int64_t w = std::min(width, p.V - v0);
    const Logits whole{weights<T, NP>(p, W, v0, w, st), Hm, p.rows, NP ? p.dp : p.d, v0, w, label,
                       NP == 2 ? static_cast<const float *>(W) + v0 * p.d : nullptr, static_cast<const float *>(H), p.d};
    const Tiling t = tiling(w, p.rows, p.d, NP);
    auto launch = [&](const Logits &a, Size size) {
      const int64_t total = tiles(size, a.width, p.rows, 1, nf, ns);
      by_alignment<NP, T>(W, p.d, [&](auto fb) {
        GCX_SHAPE(size, NP, hipLaunchKernelGGL((lse_part_kernel<P, decltype(fb)::value>), grid(total), dim3(P::Threads), 0, st, a,
                                               nf, ns, tile0, p.part, p.target, int32_t(p.V), at_once ? loss : nullptr, lse))
      });
      tile0 += nf;
    };
    launch(whole.part(0, t.first), t.size);
    if (t.first < w) launch(whole.part(t.first, w), t.then);
  }
  if (!at_once)
    hipLaunchKernelGGL(lse_join_kernel, blocks_of(ceil_div(p.rows, kJoin)), dim3(256), 0, st, p.part, p.target, label,
                       p.rows, int32_t(p.V), tile0, loss, lse);
  return launch_status();
}

template <typename T, int NP>
int launch_xent_grads(const Plan &p, const void *H, const void *W, const int32_t *label, const float *lse, const float *dloss,
                      void *dH, void *G, hipStream_t st) {
  if (p.rows == 0) {
    if (G)
      hipLaunchKernelGGL(zero_kernel<T>, dim3(unsigned(std::min<int64_t>(ceil_div(p.N * p.V * p.d, 256), 1 << 16))), dim3(256),
                         0, st, static_cast<T *>(G), p.N * p.V * p.d);
    return launch_status();
  }
  lay_out<T, NP>(H, 0, p.rows, p.d, p.dp, label, int32_t(p.V), p.H, p.hexps, st);
  constexpr int bytes = NP ? 2 : 4;
  const Matrix Hm{bytes, p.H, p.dp * bytes, p.rows * p.dp * bytes, p.hexps};
  const Matrix Pm{bytes, NP ? p.P : reinterpret_cast<char *>(p.Q), p.ld * bytes, p.rows * p.ld * bytes, nullptr};
  const Matrix Gm = NP == 2 ? Matrix{2, p.P2, p.ld * 2, p.rows * p.ld * 2, nullptr} : Pm;
  const bool at_once = p.width >= p.V && p.splits == 1 && !(NP == 1 && p.dh_size == kLarge);  // dH needs no sums
  int64_t nf, ns;
  for (int64_t v0 = 0; v0 < p.V; v0 += p.width) {
    const int64_t w = std::min(p.width, p.V - v0);
    const Matrix Wm = weights<T, NP>(p, W, v0, w, st);
    {
      const Logits whole{Wm, Hm, p.rows, NP ? p.dp : p.d, v0, w, label,
                         NP == 2 ? static_cast<const float *>(W) + v0 * p.d : nullptr, static_cast<const float *>(H), p.d};
      __bf16 *Pb = NP == 1 || dH ? reinterpret_cast<__bf16 *>(p.P) : nullptr;
      float *Q = NP == 0 || G ? p.Q : nullptr;
      const Tiling t = tiling(w, p.rows, p.d, NP);
      auto launch = [&](int64_t from, int64_t to, Size size) {
        const int64_t total = tiles(size, to - from, p.rows, 1, nf, ns);
        const Logits a = whole.part(from, to);
        const Probabilities b{lse, dloss, int32_t(p.V), p.ld, p.ld - from, Pb ? Pb + from : nullptr, Q ? Q + from : nullptr, p.rest};
        by_alignment<NP, T>(W, p.d, [&](auto fb) {
          GCX_SHAPE(size, NP, hipLaunchKernelGGL((p_kernel<P, decltype(fb)::value>), grid(total), dim3(P::Threads), 0, st, a, b, nf, ns))
        });
      };
      launch(0, t.first, t.size);
      if (t.first < w) launch(t.first, w, t.then);
    }
    if (dH) {
      constexpr int NPh = NP == 2 ? 3 : NP;
      Matrix Wh = Wm;
      if (NP == 2) {
        lay_out<T, NPh>(W, v0, w, p.d, p.dp, nullptr, 0, p.W3, nullptr, st);
        Wh = {2, p.W3, p.dp * 2, w * p.dp * 2, nullptr};
      }
      // Splits whose tiles do not fill eight XCDs evenly are dealt to them together: each alone would go to the first
      // ones (8 rows, 65536 x 216 fp32: 42 us, so 14).  Others do better a split at a time (4096 x 65536 x 2048 bf16: 45
      // of 3870 us; 12 rows, 65536 x 4096 fp32: 574 / 605).
      const int64_t splits = ceil_div(w, p.kper), one = tiles(p.dh_size, p.d, p.rows, 1, nf, ns);
      const int64_t together = up(one, 8) * 4 > one * 5 ? splits : 1, total = one * together;
      dim3 blocks = grid(total);
      blocks.z = unsigned(splits / together);
      by_alignment<NP, T>(W, p.d, [&](auto fb) {
        GCX_SHAPE(p.dh_size, NPh,
                  hipLaunchKernelGGL((dh_kernel<P, T, decltype(fb)::value>), blocks, dim3(P::Threads), 0, st, Pm, Wh,
                                     p.rows, w, p.d, p.dq, p.kper, v0 == 0, nf, ns, uint32_t(together), p.sum,
                                     at_once ? static_cast<T *>(dH) : nullptr, label, int32_t(p.V), p.rest))
      });
    }
    if (G && p.n <= kFewRows<T>) {
      const int64_t units = ceil_div(p.d, 16 / int64_t(sizeof(T)));
      int tx = 1;
      while (tx < 256 && tx < units) tx *= 2;
      const int entries = std::min(kFewEntries, 256 / tx * 32);
      const unsigned nx = unsigned(ceil_div(units, tx)), nv = unsigned(ceil_div(w, entries));
      auto few = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, blocks_of(int64_t(nx) * nv * p.N), dim3(256), 0, st, NP == 1 ? p.P : reinterpret_cast<char *>(p.Q),
                           p.ld, p.H, p.dp, p.rows, int(p.n), w, p.d, p.V, v0, tx, nx, nv, entries, label, p.rest,
                           static_cast<T *>(G));
      };
      p.n <= 4 ? few(g_few_kernel<NP, T, 4>) : (p.n <= 8 ? few(g_few_kernel<NP, T, 8>) : few(g_few_kernel<NP, T, kFewRows<T>>));
    } else if (G) {
      if (NP == 2) {
        const dim3 blocks(unsigned(p.N * (p.ld / 64) * ceil_div(p.n, kColumnRows)));
        hipLaunchKernelGGL(column_top_kernel, blocks, dim3(256), 0, st, p.Q, p.n, p.ld, p.top);
        hipLaunchKernelGGL(split_columns_kernel, blocks, dim3(256), 0, st, p.Q, p.rows, p.n, p.ld, p.top,
                           reinterpret_cast<_Float16 *>(p.P2));
      }
      const Size size = size_for(p.d, w, p.N, p.n, NP);
      const int64_t total = tiles(size, p.d, w, p.N, nf, ns);
      GCX_SHAPE(size, NP, hipLaunchKernelGGL((g_kernel<P, T>), grid(total), dim3(P::Threads), 0, st, Gm, Hm, p.n, w, p.ld,
                                             p.d, p.dp, p.V, v0, nf, ns, p.N, p.top, label, p.rest, static_cast<T *>(G)))
    }
  }
  if (dH && !at_once) {
    auto finish = [&](auto kernel, int each) {
      hipLaunchKernelGGL(kernel, dim3(unsigned(std::min<int64_t>(ceil_div(p.rows * (p.dq / 4), 256 / each), 1 << 14))), dim3(256), 0,
                         st, p.sum, p.rows, p.d, p.dq, int(p.splits), static_cast<const T *>(W), label, int32_t(p.V), p.rest,
                         static_cast<T *>(dH));
    };
    p.splits >= 16 ? finish(dh_finish_kernel<T, 16>, 16) : finish(dh_finish_kernel<T, 1>, 1);
  }
  return launch_status();
}

}  // namespace
}  // namespace gcx

extern "C" size_t gc_softmax_xent_workspace_size(int64_t rows, int32_t V, int64_t d, int32_t dtype) {
  using namespace gcx;
  if (rows < 1 || !xent_sizes_ok(rows, 1, V, d, dtype)) return 0;
  return plan(1, rows, V, d, dtype, false, nullptr).bytes;
}

extern "C" int gc_softmax_xent(const void *H, const void *W, const int32_t *label, int64_t rows, int32_t V, int64_t d,
                               int32_t dtype, float *loss, float *lse, void *workspace, size_t workspace_bytes,
                               hipStream_t stream) {
  using namespace gcx;
  if (!xent_sizes_ok(rows, 1, V, d, dtype)) return GC_EINVAL;
  if (rows == 0) return GC_OK;
  if (!H || !W || !label || !loss || !lse) return GC_EINVAL;
  const Plan p = plan(1, rows, V, d, dtype, false, workspace);
  if (!workspace || workspace_bytes < p.bytes || !aligned16(workspace)) return GC_EINVAL;
  const int dev = check_device();
  if (dev != GC_OK) return dev;
  (void)hipGetLastError();
  if (dtype == GC_BF16) return launch_xent<__bf16, 1>(p, H, W, label, loss, lse, stream);
  return p.NP == 0 ? launch_xent<float, 0>(p, H, W, label, loss, lse, stream)
                   : launch_xent<float, 2>(p, H, W, label, loss, lse, stream);
}

extern "C" size_t gc_softmax_xent_grads_workspace_size(int32_t N, int32_t n, int32_t V, int64_t d, int32_t dtype) {
  using namespace gcx;
  const int64_t rows = int64_t(N) * n;
  if (N < 1 || n < 1 || !xent_sizes_ok(rows, N, V, d, dtype)) return 0;
  return plan(N, n, V, d, dtype, true, nullptr).bytes;
}

extern "C" int gc_softmax_xent_grads(const void *H, const void *W, const int32_t *label, const float *lse,
                                     const float *dloss, int32_t N, int32_t n, int32_t V, int64_t d, int32_t dtype,
                                     void *dH, void *G, void *workspace, size_t workspace_bytes, hipStream_t stream) {
  using namespace gcx;
  if (N < 0 || n < 0 || !xent_sizes_ok(int64_t(N) * n, N, V, d, dtype)) return GC_EINVAL;
  if (N == 0) return GC_OK;
  if (n > 0 && (!H || !W || !label || !lse)) return GC_EINVAL;
  if (!dH && !G) return n > 0 ? GC_EINVAL : GC_OK;
  Plan p{};
  if (n > 0) {
    p = plan(N, n, V, d, dtype, true, workspace);
    if (!workspace || workspace_bytes < p.bytes || !aligned16(workspace)) return GC_EINVAL;
  } else {
    p.N = N;
    p.V = V;
    p.d = d;
  }
  const int dev = check_device();
  if (dev != GC_OK) return dev;
  (void)hipGetLastError();
  if (dtype == GC_BF16) return launch_xent_grads<__bf16, 1>(p, H, W, label, lse, dloss, dH, G, stream);
  return p.NP == 0 ? launch_xent_grads<float, 0>(p, H, W, label, lse, dloss, dH, G, stream)
                   : launch_xent_grads<float, 2>(p, H, W, label, lse, dloss, dH, G, stream);
}
