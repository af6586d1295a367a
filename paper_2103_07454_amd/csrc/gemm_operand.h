// A matrix as the products' kernels are handed it.
#pragma once
#include <stdint.h>

namespace evg {

struct GemmOperand {
  const void* p;      // null: this part is left out
  int64_t worker, ld; // elements between workers and between rows of what lies in memory
};

}  // namespace evg
