// What the operators of a language-model head share: values stored as fp32 or bf16.
#pragma once

#include <algorithm>

#include "common.h"

namespace gcx {

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__bf16 v) { return static_cast<float>(v); }
template <typename T>
__device__ __forceinline__ T from_f32(float v) {  // to nearest
  return static_cast<T>(v);
}

// A launch's blocks, in rows of the grid where they are many: a row has less than 2^32 threads (of up to 1024 a
// block), and whole eights of blocks, as they go to the XCDs.  The last row's may go past the last block.
inline dim3 blocks_of(int64_t blocks) {
  constexpr int64_t kRow = int64_t(1) << 21;
  return blocks <= kRow ? dim3(unsigned(blocks)) : dim3(unsigned(kRow), unsigned(ceil_div(blocks, kRow)));
}
__device__ __forceinline__ uint32_t block_number() { return blockIdx.y * gridDim.x + blockIdx.x; }

}  // namespace gcx
