// sizes.h -- arithmetic of sizes on the host.
#pragma once

#include <cstddef>
#include <cstdint>

namespace tg {

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline size_t round256(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace tg
