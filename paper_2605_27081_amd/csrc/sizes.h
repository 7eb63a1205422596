// Arithmetic of sizes on the host.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace remoe {

static inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
static inline size_t align_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

}  // namespace remoe
