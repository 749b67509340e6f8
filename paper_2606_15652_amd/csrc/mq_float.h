// 16- and 32-bit floating types of the operators that take more than fp16.
#pragma once

#include "mq_device.h"

namespace mq {

// Eight consecutive 16-bit values, as loaded, and as fp32.
template <typename T>
struct Vec8 {
    typedef T type __attribute__((ext_vector_type(8)));
};

template <typename T>
__device__ __forceinline__ f32x8 load8(const T* p) {
    return __builtin_convertvector(*reinterpret_cast<const typename Vec8<T>::type*>(p), f32x8);
}
template <typename T>
__device__ __forceinline__ void store8(T* p, f32x8 v) {
    *reinterpret_cast<typename Vec8<T>::type*>(p) = __builtin_convertvector(v, typename Vec8<T>::type);
}

constexpr uint32_t kFloatInf = 0x7F800000u;   // fp32 bits (sign cleared) from here on: infinity, NaN

}  // namespace mq

namespace mq_host {

inline bool is_half_type(mq_dtype t) { return t == MQ_FP16 || t == MQ_BF16; }

// f(T{}) with the 16-bit type of t (checked by the caller)
template <typename F>
inline mq_status with_half_type(mq_dtype t, F&& f) {
    if (t == MQ_FP16) return f(_Float16{});
    return f(__bf16{});
}

}  // namespace mq_host
