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

// A launch has fewer than 2^32 threads in x: f(first, count) launches workgroups first .. first + count of the `blocks` that the sizes call for.
template <typename F>
static inline int launch_parts(int64_t blocks, int64_t threads, F f) {
    const int64_t most = ((int64_t)1 << 31) / threads;
    for (int64_t first = 0; first < blocks; first += most) {
        f(first, std::min(most, blocks - first));
        HIP_TRY(hipGetLastError());
    }
    return HAG_OK;
}

// 16 bytes of a row: memory operations of that width at any address that suits one element, which gfx950's global loads and stores take.
template <typename T>
constexpr int kVec = 16 / (int)sizeof(T);
template <typename T>
struct VecOf {
    typedef T type __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
};

// p[0 .. kVec) as it comes from memory.  Where not all of it is memory of the matrix (`readable`), the first `have` elements, the others 0.
template <typename T>
__device__ __forceinline__ typename VecOf<T>::type load_vec(const T *p, bool readable, int have) {
    typename VecOf<T>::type raw = {};
    if (readable) {
        raw = *reinterpret_cast<const typename VecOf<T>::type *>(p);
    } else {
#pragma unroll
        for (int e = 0; e < kVec<T>; ++e)
            if (e < have) raw[e] = p[e];
    }
    return raw;
}
template <typename T>
__device__ __forceinline__ typename VecOf<T>::type load_vec(const T *p) { return *reinterpret_cast<const typename VecOf<T>::type *>(p); }

// p[0 .. min(have, kVec)) = v, each rounded once.  STREAM: written past the caches' order of use, so that what was read stays there rather than what is written.
template <bool STREAM = false, typename T>
__device__ __forceinline__ void store_vec(T *p, int have, const float (&v)[kVec<T>]) {
    if (have >= kVec<T>) {
        typename VecOf<T>::type raw;
#pragma unroll
        for (int e = 0; e < kVec<T>; ++e) raw[e] = (T)v[e];
        if (STREAM) __builtin_nontemporal_store(raw, reinterpret_cast<typename VecOf<T>::type *>(p));
        else *reinterpret_cast<typename VecOf<T>::type *>(p) = raw;
    } else {
#pragma unroll
        for (int e = 0; e < kVec<T>; ++e)
            if (e < have) p[e] = (T)v[e];
    }
}

// The same into a row of fp32, whatever the vector's length.
template <typename O, int V>
__device__ __forceinline__ void store_cols(O *p, int have, const float (&v)[V]) {
    if constexpr (V == kVec<O>) {
        store_vec(p, have, v);
    } else {
#pragma unroll
        for (int q = 0; q < V; q += kVec<O>) {
            float part[kVec<O>];
#pragma unroll
            for (int e = 0; e < kVec<O>; ++e) part[e] = v[q + e];
            store_vec(p + q, have - q, part);
        }
    }
}

// Columns col .. col + kVec of the row at element `at` of a matrix whose last row ends at `extent`; lanes beyond the row's end get its first ones, so that no load waits for a
// condition.  TAIL: d is no multiple of the vector, a row's last vector brings elements of the next row along, and at the end of the matrix is read element by element.
template <typename T, bool TAIL>
__device__ __forceinline__ typename VecOf<T>::type load_columns(const T *base, int64_t at, int col, int d, int64_t extent) {
    const T *p = base + at + (col < d ? col : 0);
    return TAIL ? load_vec(p, p - base + kVec<T> <= extent, d - col) : load_vec(p);
}

template <int CTRL>
__device__ __forceinline__ float dpp_move(float v) {
    return __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, true));
}
typedef unsigned elem_u2_t __attribute__((ext_vector_type(2)));

// Sum over groups of W adjacent lanes (a power of two), in every lane of the group: moves within a row of 16 lanes, then swaps of rows and of halves.
template <int W>
__device__ __forceinline__ float lanes_sum(float v) {
    if (W > 1) v += dpp_move<0xB1>(v);                     // lane ^ 1
    if (W > 2) v += dpp_move<0x4E>(v);                     // lane ^ 2
    if (W > 4) v += dpp_move<0x141>(v);                    // the other four of eight
    if (W > 8) v += dpp_move<0x140>(v);                    // the other eight of sixteen
    if (W > 16) {
        const elem_u2_t s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(s.x) + __uint_as_float(s.y);
    }
    if (W > 32) {
        const elem_u2_t s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(s.x) + __uint_as_float(s.y);
    }
    return v;
}

}  // namespace hag
