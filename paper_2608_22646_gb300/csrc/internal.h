// What the translation units of libcai.so share besides the C ABI.
#pragma once

#include <cstddef>

namespace cai {

// cudaMalloc as a status code, counted by cai_test_fail_alloc_after.
int device_alloc(void** p, size_t bytes);

}  // namespace cai
