// Rows of the training operators: fp32, fp16 or bf16 in memory, fp32 in registers.
#pragma once

#include "common.h"

namespace sa {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

// A value as it is in memory; to fewer bits by one rounding to nearest even.
template <class T>
__device__ inline float load_elem(const T *p) { return (float)*p; }
template <class T>
__device__ inline void store_elem(T *p, float v) { *p = (T)v; }

// What a launch does with the type of a residual stream (X) and of the rows it meets (Y).
template <template <class, class> class F, class... A>
int for_row_types(int x_type, int y_type, A &&...a) {
    if (x_type == SA_F32 && y_type == SA_F32) return F<float, float>::run(a...);
    if (x_type == SA_F32 && y_type == SA_F16) return F<float, f16_t>::run(a...);
    if (x_type == SA_F32 && y_type == SA_BF16) return F<float, bf16_t>::run(a...);
    if (x_type == SA_F16) return F<f16_t, f16_t>::run(a...);
    return F<bf16_t, bf16_t>::run(a...);
}

inline int check_row_types(const char *what, int x_type, int y_type) {
    SA_REQUIRE(x_type >= SA_F32 && x_type <= SA_BF16 && y_type >= SA_F32 && y_type <= SA_BF16, SA_ERR_INVALID,
               "%s: unknown element type (%d, %d)", what, x_type, y_type);
    SA_REQUIRE(x_type == y_type || x_type == SA_F32, SA_ERR_UNSUPPORTED,
               "%s: element types %d and %d do not go together (the same, or a residual stream of SA_F32)", what, x_type, y_type);
    return SA_OK;
}

}  // namespace sa
