// Whole numbers divided by one that a launch knows, with a product.
#pragma once
#include <hip/hip_runtime.h>
#include <cstdint>

namespace ppd {

// x / size for x below 2^31, size 1 .. 2^30.  With 2^(s - 1) < size <= 2^s, m = floor(2^(31 + s) / size) + 1: m size is above 2^(31 + s) by at most size <= 2^s, so that
// x m / 2^(31 + s) is above x / size by at most x / (size 2^31), less than what parts x / size from the next whole number.
struct Divider {
  uint32_t by, shift;
  Divider() : by(0), shift(0) {}
  explicit Divider(uint32_t size) : shift(0) {
    while ((1u << shift) < size) ++shift;
    by = (uint32_t)((((uint64_t)1 << (31 + shift)) / size) + 1);
  }
  __host__ __device__ __forceinline__ uint32_t operator()(uint32_t x) const { return (uint32_t)((uint64_t)(2u * x) * by >> 32) >> shift; }
};

}  // namespace ppd
