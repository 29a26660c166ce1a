// Host driver for the sanitizer build of libgcx: the language-model head's entry points, as abi_validate.cpp has the
// others.  Workspace queries over a grid of sizes up to the types' ends, argument validation, sizes whose buffers could
// not exist, and valid calls up to the device check (no device: a non-OK status, nothing launched).
#include <cstdint>
#include <cstdio>
#include <limits>

#include "gcx.h"

static int failures = 0;

#define CHECK(cond)                                                           \
  do {                                                                        \
    if (!(cond)) {                                                            \
      std::fprintf(stderr, "check failed at line %d: %s\n", __LINE__, #cond); \
      ++failures;                                                             \
    }                                                                         \
  } while (0)

static void *const p = reinterpret_cast<void *>(uintptr_t(256));  // never dereferenced
static const float *const fp = static_cast<const float *>(p);
static float *const fo = static_cast<float *>(p);
static const int32_t *const ip = static_cast<const int32_t *>(p);
static const int64_t H = std::numeric_limits<int64_t>::max(), L = std::numeric_limits<int64_t>::min();
static const int32_t H32 = std::numeric_limits<int32_t>::max(), L32 = std::numeric_limits<int32_t>::min();
static const size_t Z = std::numeric_limits<size_t>::max();

// every size and plan that the queries and the calls form, refused or not
static void sizes() {
  const int32_t ns[] = {L32, -1, 0, 1, 7, 16, 17, 512, 65537, 1 << 24, H32};
  const int64_t ds[] = {L, -1, 0, 1, 9, 1000, 16392, 1 << 20, (1 << 20) + 1, int64_t(1) << 33, int64_t(1) << 40, H};
  const int32_t vs[] = {L32, 0, 1, 129, 131072, 1 << 28, H32};
  const int64_t rows[] = {L, -1, 0, 1, 160, 161, 4096, int64_t(1) << 28, int64_t(1) << 31, (int64_t(1) << 31) + 1, H};
  for (int64_t d : ds) {
    for (int32_t N : ns)
      for (int32_t n : ns) {
        const size_t norm = gc_layer_norm_grads_workspace_size(N, n, d);
        CHECK(norm == 0 || (N > 0 && n > 0 && d > 0));
        if (norm > 0)
          CHECK(gc_layer_norm_grads(p, p, fp, fp, fp, N, n, d, GC_F32, p, fo, fo, p, norm - 1, nullptr) == GC_EINVAL);
        else if (N > 0)
          CHECK(gc_layer_norm_grads(p, p, fp, fp, fp, N, n, d, GC_BF16, p, fo, fo, p, Z, nullptr) != GC_OK);
        for (int32_t V : vs)
          for (int32_t t = GC_F32; t <= GC_BF16; ++t) {
            const size_t need = gc_softmax_xent_grads_workspace_size(N, n, V, d, t);
            CHECK(need == 0 || (N > 0 && n > 0 && V > 0 && d > 0));
            if (need > 0)
              CHECK(gc_softmax_xent_grads(p, p, ip, fp, fp, N, n, V, d, t, p, p, p, need - 1, nullptr) == GC_EINVAL);
            else if (N > 0)
              CHECK(gc_softmax_xent_grads(p, p, ip, fp, fp, N, n, V, d, t, p, p, p, Z, nullptr) != GC_OK);
          }
      }
    for (int64_t r : rows) {
      CHECK((r == 0 && d > 0 && d <= int64_t(1) << 40) == (gc_layer_norm(p, fp, fp, r, d, 0.0, GC_F32, p, fo, fo, nullptr) == GC_OK));
      CHECK((r == 0 && d > 0 && d <= int64_t(1) << 32) == (gc_dropout(p, p, r, d, 0.5, 1, 0, 0, GC_BF16, p, nullptr) == GC_OK));
      for (int32_t V : vs)
        for (int32_t t = GC_F32; t <= GC_BF16; ++t) {
          const size_t need = gc_softmax_xent_workspace_size(r, V, d, t);
          CHECK(need == 0 || (r > 0 && V > 0 && d > 0));
          if (need > 0) CHECK(gc_softmax_xent(p, p, ip, r, V, d, t, fo, fo, p, need - 1, nullptr) == GC_EINVAL);
          else if (r != 0) CHECK(gc_softmax_xent(p, p, ip, r, V, d, t, fo, fo, p, Z, nullptr) != GC_OK);
        }
    }
  }
}

static void validation() {
  const int E = GC_EINVAL;
  // dropout
  CHECK(gc_dropout(nullptr, p, 4, 8, 0.1, 1, 0, 0, GC_F32, p, nullptr) == E);
  CHECK(gc_dropout(p, p, 4, 8, 0.1, 1, 0, 0, GC_F32, nullptr, nullptr) == E);
  CHECK(gc_dropout(p, p, 4, 8, 0.1, 1, 0, 0, 2, p, nullptr) == E);
  CHECK(gc_dropout(p, p, 4, 8, -0.1, 1, 0, 0, GC_F32, p, nullptr) == E);
  CHECK(gc_dropout(p, p, 4, 8, 1.1, 1, 0, 0, GC_F32, p, nullptr) == E);
  CHECK(gc_dropout(p, p, 4, 8, std::numeric_limits<double>::quiet_NaN(), 1, 0, 0, GC_F32, p, nullptr) == E);
  CHECK(gc_dropout(p, p, 4, 8, 0.1, 1, 0, -1, GC_F32, p, nullptr) == E);
  CHECK(gc_dropout(p, p, 4, 8, 0.1, ~uint64_t(0), ~uint32_t(0), H, 9, p, nullptr) == E);
  CHECK(gc_dropout(nullptr, nullptr, 0, 8, 0.1, 1, 0, 0, GC_F32, nullptr, nullptr) == GC_OK);
  // layer norm
  CHECK(gc_layer_norm(nullptr, fp, fp, 4, 8, 1e-5, GC_F32, p, fo, fo, nullptr) == E);
  CHECK(gc_layer_norm(p, fp, fp, 4, 8, 1e-5, GC_F32, p, nullptr, fo, nullptr) == E);
  CHECK(gc_layer_norm(p, fp, fp, 4, 8, 1e-5, GC_F32, p, fo, nullptr, nullptr) == E);
  CHECK(gc_layer_norm(p, fp, fp, 4, 8, -1e-5, GC_F32, p, fo, fo, nullptr) == E);
  CHECK(gc_layer_norm(p, fp, fp, 4, 8, std::numeric_limits<double>::quiet_NaN(), GC_F32, p, fo, fo, nullptr) == E);
  CHECK(gc_layer_norm(p, fp, fp, 4, 8, 1e-5, 7, p, fo, fo, nullptr) == E);
  const size_t norm = gc_layer_norm_grads_workspace_size(3, 400, 64);
  CHECK(norm > 0);
  CHECK(gc_layer_norm_grads(p, p, fp, fp, fp, 3, 400, 64, GC_F32, p, fo, fo, nullptr, norm, nullptr) == E);
  CHECK(gc_layer_norm_grads(p, p, fp, fp, fp, 3, 400, 64, GC_F32, p, fo, fo, static_cast<char *>(p) + 4, norm, nullptr) == E);
  CHECK(gc_layer_norm_grads(p, nullptr, fp, fp, fp, 3, 400, 64, GC_F32, p, fo, fo, p, norm, nullptr) == E);
  CHECK(gc_layer_norm_grads(p, p, fp, fp, fp, 3, 400, 64, GC_F32, nullptr, nullptr, nullptr, p, norm, nullptr) == E);
  CHECK(gc_layer_norm_grads(p, p, fp, fp, fp, 0, 400, 64, GC_F32, p, fo, fo, p, norm, nullptr) == GC_OK);
  // softmax cross entropy
  for (int32_t t = GC_F32; t <= GC_BF16; ++t) {
    const size_t a = gc_softmax_xent_workspace_size(6, 100, 64, t), b = gc_softmax_xent_grads_workspace_size(2, 3, 100, 64, t);
    CHECK(a > 0 && b > 0);
    CHECK(gc_softmax_xent(p, nullptr, ip, 6, 100, 64, t, fo, fo, p, a, nullptr) == E);
    CHECK(gc_softmax_xent(p, p, nullptr, 6, 100, 64, t, fo, fo, p, a, nullptr) == E);
    CHECK(gc_softmax_xent(p, p, ip, 6, 100, 64, t, nullptr, fo, p, a, nullptr) == E);
    CHECK(gc_softmax_xent(p, p, ip, 6, 100, 64, t, fo, fo, nullptr, a, nullptr) == E);
    CHECK(gc_softmax_xent(p, p, ip, 6, 100, 64, t, fo, fo, static_cast<char *>(p) + 8, a, nullptr) == E);
    CHECK(gc_softmax_xent(p, p, ip, 0, 100, 64, t, fo, fo, nullptr, 0, nullptr) == GC_OK);
    CHECK(gc_softmax_xent_grads(p, p, ip, nullptr, fp, 2, 3, 100, 64, t, p, p, p, b, nullptr) == E);
    CHECK(gc_softmax_xent_grads(p, p, ip, fp, nullptr, 2, 3, 100, 64, t, nullptr, nullptr, p, b, nullptr) == E);
    CHECK(gc_softmax_xent_grads(p, p, ip, fp, nullptr, 2, 3, 100, 64, t, p, p, nullptr, b, nullptr) == E);
    CHECK(gc_softmax_xent_grads(p, p, ip, fp, nullptr, 0, 3, 100, 64, t, p, p, nullptr, 0, nullptr) == GC_OK);
  }
  CHECK(gc_softmax_xent(p, p, ip, 6, 100, 64, 2, fo, fo, p, Z, nullptr) == E);
  CHECK(gc_softmax_xent_grads(p, p, ip, fp, fp, 2, 3, 100, 64, -1, p, p, p, Z, nullptr) == E);
}

static void device_check_without_gpu() {
  CHECK(gc_dropout(p, p, 4, 8, 0.1, 1, 0, 0, GC_F32, p, nullptr) != GC_OK);
  CHECK(gc_layer_norm(p, fp, fp, 4, 8, 1e-5, GC_BF16, p, fo, fo, nullptr) != GC_OK);
  CHECK(gc_layer_norm_grads(p, p, fp, fp, fp, 3, 400, 64, GC_F32, p, fo, fo, p, Z, nullptr) != GC_OK);
  CHECK(gc_softmax_xent(p, p, ip, 6, 100, 64, GC_F32, fo, fo, p, Z, nullptr) != GC_OK);
  CHECK(gc_softmax_xent_grads(p, p, ip, fp, fp, 2, 3, 100, 64, GC_BF16, p, p, p, Z, nullptr) != GC_OK);
  CHECK(gc_softmax_xent_grads(p, p, ip, fp, fp, 2, 0, 100, 64, GC_F32, nullptr, p, nullptr, 0, nullptr) != GC_OK);
}

int main() {
  sizes();
  validation();
  device_check_without_gpu();
  if (failures) {
    std::fprintf(stderr, "%d checks failed\n", failures);
    return 1;
  }
  std::printf("ok\n");
  return 0;
}
