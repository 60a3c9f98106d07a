// What the training operators' host code shares that needs no HIP.
#ifndef DEAR_OPS_SIZES_H
#define DEAR_OPS_SIZES_H

#include <cstdint>

namespace dear_ops {

// HIP takes fewer than 2^32 threads along a dimension of a launch.
constexpr int64_t MAX_THREADS = 0xffffffff;

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace dear_ops
#endif
