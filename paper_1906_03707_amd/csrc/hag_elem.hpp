// Matrix elements of 32 and 16 bits for the kernels that compute in fp32 whatever they read and write (lookups, layer norm, clipping).
#pragma once
#include "hag_device_common.hpp"

namespace hag {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

static inline bool elem_type(hag_dtype_t t) { return t == HAG_F32 || t == HAG_BF16 || t == HAG_F16; }
static inline int elem_size(hag_dtype_t t) { return t == HAG_F32 ? 4 : 2; }

// Calls f with a value of the element type: elem_switch(dtype, [&](auto e) { using T = decltype(e); ... }).
template <typename F>
static inline int elem_switch(hag_dtype_t t, F f) {
    return t == HAG_F32 ? f(float()) : t == HAG_BF16 ? f(bf16_t()) : f(f16_t());
}
// An int64_t or int32_t array of ids.
template <typename F>
static inline int id_switch(hag_dtype_t t, F f) {
    return t == HAG_I64 ? f(int64_t()) : f(int32_t());
}

}  // namespace hag
