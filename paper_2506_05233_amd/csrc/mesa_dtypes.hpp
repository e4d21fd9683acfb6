// Element types (MESA_DTYPE_*); no GPU types, so that host code can be compiled without one.
#pragma once

namespace mesa {

constexpr int kF32 = 0, kBf16 = 1, kQ8 = 2;

}  // namespace mesa
