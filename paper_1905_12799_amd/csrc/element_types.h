// Arrays of fp32, bf16 or fp16: what a kernel reads is widened to fp32, what it writes is rounded once, to nearest even.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rls.h"

namespace rls {

template <typename T>
struct Vec4 {
    using type __attribute__((ext_vector_type(4))) = T;
};
template <typename T>
using vec4 = typename Vec4<T>::type;
template <typename T>
struct Vec8 {
    using type __attribute__((ext_vector_type(8))) = T;
};
template <typename T>
using vec8 = typename Vec8<T>::type;

inline bool is_type(int32_t type) { return type == RLS_F32 || type == RLS_BF16 || type == RLS_F16; }
inline int type_bytes(int32_t type) { return type == RLS_F32 ? 4 : 2; }

}  // namespace rls
