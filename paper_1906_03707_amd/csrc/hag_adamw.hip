// A step of AdamW over many tensors, with their states in 32 bits or in 8.
//   g' = c g, c = min(1, max_norm / norm);  m' = b1 m + (1 - b1) g',  v' = b2 v + (1 - b2) g'^2
//   p' = p (1 - lr decay) - lr / (1 - b1^t) m' / (sqrt(v' / (1 - b2^t)) + eps)
// In 8 bits m and the root r of v are kept, in blocks of 32 consecutive elements with a power of two each (hag_fp8.hpp); the parameters take m' and r' as they were before they are rounded.
// Rounded to the nearest they would never move: a step changes r by a part of 5e-4 at b2 = 0.999, half a step of 3 mantissa bits is a part of 0.03 to 0.06.  So both are rounded up
// with the probability that is the part cut off, by 16 bits of a hash of seed, step and element, which keeps the mean whatever the sequence of gradients.  A root that is not zero does
// not become zero, which would leave m' / eps.
#include "hag_fp8.hpp"

#include <cmath>

namespace hag {

// The tensors are cut into units of at most `unit` elements, one workgroup each; a launch takes as many tensors as its argument block holds.
constexpr int kAdamTensors = 48;
constexpr int64_t kAdamUnits = 4096, kAdamRound = 1024;
struct AdamArgs {
    struct Tensor {
        void *param;
        const void *grad;
        void *m, *v, *copy;
        uint8_t *m_scales, *v_scales;
        int64_t count;
        int32_t types;               // param, grad, copy in 8 bits each
        int32_t first_unit;          // of this launch
    } t[kAdamTensors];
    int64_t unit;
    int32_t tensors, units;
    double lr, beta1, beta2, eps, decay, max_norm;
    const float *lr_at, *norm;       // or NULL
    const int64_t *step_at;          // or NULL
    int64_t step;
    uint32_t seed;
};
static_assert(sizeof(AdamArgs) <= 4032, "kernel arguments are limited to 4 KB");

// 32 bits that depend on all of x: two rounds of a shifted exclusive or and a product with the fraction bits of sqrt(2), sqrt(3)
__host__ __device__ __forceinline__ uint32_t mixed(uint32_t x) {
    x = (x ^ (x >> 15)) * 0x6a09e667u;
    x = (x ^ (x >> 13)) * 0xbb67ae85u;
    return x ^ (x >> 16);
}

// b^t by squaring: off by t roundings of 64 bits where the power is not negligible
__device__ __forceinline__ double power(double b, int64_t t) {
    double p = 1.;
    for (; t > 0; t >>= 1, b *= b)
        if (t & 1) p *= b;
    return p;
}

struct AdamNumbers {
    float clip, clip_rest;                                 // the factor is (clip + clip_rest) * 2^clip_exponent, clip in [1/2, 1]: their products with a gradient are rounded once
    int clip_exponent;
    float b1, a1, b2, a2, keep, rate, root, eps;           // a: 1 - b;  keep: 1 - lr decay, rate: lr / (1 - b1^t), root: 1 / sqrt(1 - b2^t)
    uint32_t key;
};

// Four elements: of 32 bits 16 bytes, of 16 bits 8, of 8 bits 4, at any address that suits one element
template <typename T>
struct Four {
    typedef T type __attribute__((ext_vector_type(4), aligned(sizeof(T))));
};
template <typename T>
__device__ __forceinline__ typename Four<T>::type load4(const T *p, int have) {
    typename Four<T>::type raw = {};
    if (have >= 4) {
        raw = *reinterpret_cast<const typename Four<T>::type *>(p);
    } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < have) raw[e] = p[e];
    }
    return raw;
}
template <typename T>
__device__ __forceinline__ void store4(T *p, int have, const float (&v)[4]) {
    if (have >= 4) {
        typename Four<T>::type raw;
#pragma unroll
        for (int e = 0; e < 4; ++e) raw[e] = (T)v[e];
        *reinterpret_cast<typename Four<T>::type *>(p) = raw;
    } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < have) p[e] = (T)v[e];
    }
}
__device__ __forceinline__ void store_codes(uint8_t *p, int have, uint32_t codes) {
    typedef uint32_t word_t __attribute__((aligned(1)));
    if (have >= 4) {
        *reinterpret_cast<word_t *>(p) = codes;
    } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < have) p[e] = (uint8_t)(codes >> 8 * e);
    }
}
__device__ __forceinline__ uint32_t load_codes(const uint8_t *p, int have) {
    typedef uint32_t word_t __attribute__((aligned(1)));
    if (have >= 4) return *reinterpret_cast<const word_t *>(p);
    uint32_t codes = 0;
#pragma unroll
    for (int e = 0; e < 3; ++e)
        if (e < have) codes |= (uint32_t)p[e] << 8 * e;
    return codes;
}
__device__ __forceinline__ void decode4(uint32_t codes, uint32_t byte, float (&v)[4]) {
    typedef float pair_t __attribute__((ext_vector_type(2)));
    const pair_t a = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
    const float scale = __uint_as_float(byte << 23 | (byte == 0 || byte == 255 ? 1u << 22 : 0u));       // 2^-127 is below the ordinary numbers, 255 is none
    v[0] = a.x * scale;
    v[1] = a.y * scale;
    v[2] = b.x * scale;
    v[3] = b.y * scale;
}

// The amount of an element in 8 bits, rounded up where its 16 random bits and a half (`random`, 16 times as much) and the part that is cut off, in 2^-16 of a step, make more than a step.
// |v| / scale as a float of an exponent bias of 7 instead of 127 is |v| / scale * 2^-120, whose upper bits then are the element's.
__device__ __forceinline__ uint32_t dithered(float v, uint32_t byte, uint32_t random) {
    return (__float_as_uint(ldexpf(fabsf(v), 7 - (int)byte)) + random) >> 20;         // 127 - byte - 120
}

// Squares below 2^-126 have a root that counts where eps is smaller still, and the hardware's root takes them for zeros: numbers below 2^-96 are taken times 2^64, their roots times 2^-32,
// both exact.
constexpr float kRootLeast = 0x1p-96f, kRootUp = 0x1p64f, kRootBack = 0x1p-32f;
__device__ __forceinline__ float near_root(float x) {
    const bool least = x < kRootLeast;
    return __builtin_amdgcn_sqrtf(least ? x * kRootUp : x) * (least ? kRootBack : 1.f);
}
// The root rounded correctly, as IEEE's, by Tuckerman's test: s is right if s (s - u) < x <= s (s + u) for the numbers s - u and s + u beside it, and the hardware's is at most one of them off.
__device__ __forceinline__ float root_of(float x) {
    const bool least = x < kRootLeast;
    const float of = least ? x * kRootUp : x, s = __builtin_amdgcn_sqrtf(of), down = __uint_as_float(__float_as_uint(s) - 1u), up = __uint_as_float(__float_as_uint(s) + 1u);
    float r = fmaf(-down, s, of) <= 0.f ? down : s;        // (of zero, infinity and no number: comparisons with no number, s stays)
    r = fmaf(-up, s, of) > 0.f ? up : r;
    return r * (least ? kRootBack : 1.f);
}

// Four elements of a tensor, `have` of them there (FULL: all), as they come from memory: elements at + mine and on, `at` the workgroup's, a multiple of 1024.  Eight adjacent lanes have a
// block's.
template <typename P, typename G, int BITS, bool FULL>
struct AdamFour {
    int64_t at;
    uint32_t mine;
    int have;
    typename Four<P>::type p;
    typename Four<G>::type g;
    typename Four<float>::type m, v;
    uint32_t m_codes, v_codes, m_byte, v_byte;

    __device__ __forceinline__ void load(const AdamArgs::Tensor &t, int64_t first, uint32_t lane, int there) {
        at = first;
        mine = lane;
        have = FULL ? 4 : there;
        p = load4((const P *)t.param + at + mine, have);
        g = load4((const G *)t.grad + at + mine, have);
        if (BITS == 32) {
            m = load4((const float *)t.m + at + mine, have);
            v = load4((const float *)t.v + at + mine, have);
            return;
        }
        const bool in = have > 0;
        m_codes = load_codes((const uint8_t *)t.m + at + mine, have);
        v_codes = load_codes((const uint8_t *)t.v + at + mine, have);
        m_byte = in ? (t.m_scales + at / kScaleBlock)[mine / kScaleBlock] : 127u;
        v_byte = in ? (t.v_scales + at / kScaleBlock)[mine / kScaleBlock] : 127u;
    }

    __device__ __forceinline__ void step(const AdamArgs::Tensor &t, const AdamNumbers &a) {
// what the 8-bit states are rounded from is the same everywhere, whatever is fused: products and sums are rounded one by one
#pragma clang fp contract(off)
        float nm[4], nv[4], np[4];
        if (BITS == 8) {
            decode4(m_codes, m_byte, nm);
            decode4(v_codes, v_byte, nv);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float d = ldexpf(fmaf((float)g[e], a.clip, (float)g[e] * a.clip_rest), a.clip_exponent);
            nm[e] = a.b1 * (BITS == 8 ? nm[e] : m[e]) + a.a1 * d;
            float root;
            if (BITS == 8) {
                root = nv[e] = root_of(a.b2 * (nv[e] * nv[e]) + a.a2 * (d * d));
            } else {
                nv[e] = a.b2 * v[e] + a.a2 * (d * d);
                root = near_root(nv[e]);                   // (one unit in the last place, as the reciprocal)
            }
            np[e] = fmaf(-a.rate, nm[e] * __builtin_amdgcn_rcpf(fmaf(root, a.root, a.eps)), (float)p[e] * a.keep);
        }
        store4((P *)t.param + at + mine, have, np);
        if (t.copy) {
            const int copy = t.types >> 16 & 0xff;
            if (copy == HAG_BF16) store4((bf16_t *)t.copy + at + mine, have, np);
            else if (copy == HAG_F16) store4((f16_t *)t.copy + at + mine, have, np);
            else store4((float *)t.copy + at + mine, have, np);
        }
        if (BITS == 32) {
            store4((float *)t.m + at + mine, have, nm);
            store4((float *)t.v + at + mine, have, nv);
            return;
        }
        // the largest amounts, and whether all are numbers: as whole numbers, those that are none are above all others (roots have no sign)
        uint32_t most_m = 0, most_v = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (!FULL && e >= have) nm[e] = nv[e] = 0.f;
            most_m = max(most_m, __float_as_uint(nm[e]) & 0x7fffffffu);
            most_v = max(most_v, __float_as_uint(nv[e]));
        }
        const bool numbers = max(most_m, most_v) < 0x7f800000u;
        uint32_t none = 0;                                 // bits of m's and v's elements that are none
        if (__any(!numbers)) {
            most_m = most_v = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (!(fabsf(nm[e]) < INFINITY)) { none |= 1u << e; nm[e] = 0.f; }
                if (!(fabsf(nv[e]) < INFINITY)) { none |= 16u << e; nv[e] = 0.f; }
                most_m = max(most_m, __float_as_uint(nm[e]) & 0x7fffffffu);
                most_v = max(most_v, __float_as_uint(nv[e]) & 0x7fffffffu);
            }
        }
        const uint32_t byte_m = scale_byte(lanes_max<8>(__uint_as_float(most_m))), byte_v = scale_byte(lanes_max<8>(__uint_as_float(most_v)));
        uint32_t codes_m = 0, codes_v = 0;
        // (multiples of the prime next to 2^32 divided by the golden ratio, Knuth's choice for multiplicative hashing; of any odd number from 2^32 on.  A piece does not cross 2^32)
        const uint32_t place = ((uint32_t)at + mine) * 0x9e3779b1u + a.key + (uint32_t)(at >> 32) * 0x85ebca6bu;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t random = mixed(place + (uint32_t)e * 0x9e3779b1u);
            codes_m |= (dithered(nm[e], byte_m, (random << 4 & 0xffff0u) | 8u) | (__float_as_uint(nm[e]) >> 24 & 0x80u)) << 8 * e;
            codes_v |= max(dithered(nv[e], byte_v, (random >> 12 & 0xffff0u) | 8u), min(__float_as_uint(nv[e]), 1u)) << 8 * e;
        }
        if (__any(none)) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (none >> e & 1) codes_m |= 0x7fu << 8 * e;
                if (none >> e & 16) codes_v |= 0x7fu << 8 * e;
            }
        }
        store_codes((uint8_t *)t.m + at + mine, have, codes_m);
        store_codes((uint8_t *)t.v + at + mine, have, codes_v);
        if (have > 0 && threadIdx.x % 8 == 0) {
            (t.m_scales + at / kScaleBlock)[mine / kScaleBlock] = (uint8_t)byte_m;
            (t.v_scales + at / kScaleBlock)[mine / kScaleBlock] = (uint8_t)byte_v;
        }
    }
};

// Pieces that a workgroup requests one after the other before it needs the first
constexpr int kAdamAsk = 2;
template <typename P, typename G, int BITS>
__device__ __forceinline__ void adam_unit(const AdamArgs::Tensor &t, const AdamNumbers &a, int64_t begin, int64_t end) {
    constexpr int kPiece = 4 * kBlock;
    const uint32_t mine = 4 * threadIdx.x;
    int64_t at = begin;
    for (; at + kAdamAsk * kPiece <= end; at += kAdamAsk * kPiece) {
        AdamFour<P, G, BITS, true> f[kAdamAsk];
#pragma unroll
        for (int u = 0; u < kAdamAsk; ++u) f[u].load(t, at + u * kPiece, mine, 4);
#pragma unroll
        for (int u = 0; u < kAdamAsk; ++u) f[u].step(t, a);
    }
    for (; at < end; at += kPiece) {
        AdamFour<P, G, BITS, false> f;
        f.load(t, at, mine, (int)max((int64_t)0, min(end - at - (int64_t)mine, (int64_t)4)));
        f.step(t, a);
    }
}

// Bound by moving parameters, gradients and states: 30 M fp32 parameters with states in 32 bits 167 us (28 bytes each, 5.0 TB/s; one or four pieces on their way 167 and 165, streaming stores
// 168), in 8 bits with bf16 gradients and copies 101 (16.1 bytes, 4.8; 80 vector instructions an element, which issue for three quarters of the time, 12 of them the hash).
template <int BITS>
__global__ __launch_bounds__(kBlock) void adamw_kernel(AdamArgs a) {
    AdamNumbers s;
    s.clip = 1.f;
    s.clip_rest = 0.f;
    s.clip_exponent = 0;
    if (a.norm) {
        const float norm = *a.norm;
        if (!(fabsf(norm) < INFINITY)) return;             // nothing changes
        if (norm > a.max_norm) {
            const double factor = frexp(a.max_norm / norm, &s.clip_exponent);
            s.clip = (float)factor;
            s.clip_rest = (float)(factor - s.clip);
        }
    }
    const double lr = a.lr_at ? (double)*a.lr_at : a.lr;
    const int64_t step = a.step_at ? *a.step_at : a.step;
    s.b1 = (float)a.beta1;
    s.a1 = (float)(1. - a.beta1);
    s.b2 = (float)a.beta2;
    s.a2 = (float)(1. - a.beta2);
    s.keep = (float)(1. - lr * a.decay);
    s.rate = (float)(lr / (1. - power(a.beta1, step)));
    s.root = (float)(1. / sqrt(1. - power(a.beta2, step)));
    s.eps = (float)a.eps;
    s.key = mixed(a.seed + (uint32_t)step * 0x9e3779b1u);
    int lo = 0, hi = a.tensors;                            // the tensor of this unit: the last one that does not begin after it
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.t[mid].first_unit <= (int)blockIdx.x) lo = mid; else hi = mid;
    }
    const AdamArgs::Tensor t = a.t[lo];
    const int64_t begin = (int64_t)((int)blockIdx.x - t.first_unit) * a.unit, end = min(begin + a.unit, t.count);
    switch (t.types & 0xffff) {
    case HAG_F32 | HAG_F32 << 8: adam_unit<float, float, BITS>(t, s, begin, end); break;
    case HAG_F32 | HAG_BF16 << 8: adam_unit<float, bf16_t, BITS>(t, s, begin, end); break;
    case HAG_F32 | HAG_F16 << 8: adam_unit<float, f16_t, BITS>(t, s, begin, end); break;
    case HAG_BF16 | HAG_BF16 << 8: adam_unit<bf16_t, bf16_t, BITS>(t, s, begin, end); break;
    default: adam_unit<f16_t, f16_t, BITS>(t, s, begin, end); break;
    }
}

}  // namespace hag

using namespace hag;

extern "C" {

int hag_adamw(int64_t tensors, const hag_adamw_tensor_t *list, const hag_adamw_options_t *o, void *stream) {
    if (tensors < 0 || tensors > (1 << 24)) { set_error("number of tensors must be in 0 .. 2^24"); return HAG_EINVAL; }
    if (!o || (tensors > 0 && !list)) { set_error("NULL pointer"); return HAG_EINVAL; }
    if (o->bits != 32 && o->bits != 8) { set_error("states have 32 or 8 bits"); return HAG_EINVAL; }
    if (!(o->beta1 >= 0. && o->beta1 < 1.) || !(o->beta2 >= 0. && o->beta2 < 1.)) { set_error("beta1 and beta2 must be in [0, 1)"); return HAG_EINVAL; }
    if (!(o->eps >= 0x1p-126 && o->eps <= 0x1p100)) { set_error("eps must be a positive fp32 number"); return HAG_EINVAL; }
    if (!o->lr_device && !(std::fabs(o->lr) < INFINITY)) { set_error("lr must be a number"); return HAG_EINVAL; }
    if (!(std::fabs(o->weight_decay) < INFINITY)) { set_error("weight_decay must be a number"); return HAG_EINVAL; }
    if (!o->step_device && o->step < 1) { set_error("steps count from 1"); return HAG_EINVAL; }
    if (o->norm && !(o->max_norm > 0.)) { set_error("max_norm must be positive"); return HAG_EINVAL; }
    int64_t total = 0;
    for (int64_t i = 0; i < tensors; ++i) {
        const hag_adamw_tensor_t &t = list[i];
        if (t.count < 0 || t.count > ((int64_t)1 << 48)) { set_error("count of a tensor out of range"); return HAG_EINVAL; }
        if (!elem_type((hag_dtype_t)t.param_dtype) || !elem_type((hag_dtype_t)t.grad_dtype) || (t.param_dtype != HAG_F32 && t.grad_dtype != t.param_dtype)) {
            set_error("parameters are HAG_F32, HAG_BF16 or HAG_F16, gradients have their type or, of HAG_F32 parameters, any of these");
            return HAG_EINVAL;
        }
        if (t.copy && !elem_type((hag_dtype_t)t.copy_dtype)) { set_error("a copy is HAG_F32, HAG_BF16 or HAG_F16"); return HAG_EINVAL; }
        if (t.count > 0 && (!t.param || !t.grad || !t.m || !t.v || (o->bits == 8 && (!t.m_scales || !t.v_scales)))) { set_error("NULL pointer"); return HAG_EINVAL; }
        total += t.count;
        if (total > ((int64_t)1 << 60)) { set_error("count of a tensor out of range"); return HAG_EINVAL; }
    }
    const int64_t unit = std::max<int64_t>(1, (total + kAdamUnits * kAdamRound - 1) / (kAdamUnits * kAdamRound)) * kAdamRound;
    for (int64_t i = 0; i < tensors;) {
        AdamArgs a;
        a.unit = unit;
        a.tensors = a.units = 0;
        for (; i < tensors && a.tensors < kAdamTensors; ++i) {
            const hag_adamw_tensor_t &t = list[i];
            if (t.count == 0) continue;
            a.t[a.tensors++] = {t.param, t.grad, t.m, t.v, t.copy, t.m_scales, t.v_scales, t.count, t.param_dtype | t.grad_dtype << 8 | (t.copy ? t.copy_dtype : 0) << 16, a.units};
            a.units += (int32_t)((t.count + unit - 1) / unit);
        }
        if (a.units == 0) break;
        a.lr = o->lr;
        a.beta1 = o->beta1;
        a.beta2 = o->beta2;
        a.eps = o->eps;
        a.decay = o->weight_decay;
        a.max_norm = o->max_norm;
        a.lr_at = o->lr_device;
        a.norm = o->norm;
        a.step_at = o->step_device;
        a.step = o->step;
        a.seed = o->seed;
        if (o->bits == 8) hipLaunchKernelGGL(adamw_kernel<8>, dim3((unsigned)a.units), dim3(kBlock), 0, (hipStream_t)stream, a);
        else hipLaunchKernelGGL(adamw_kernel<32>, dim3((unsigned)a.units), dim3(kBlock), 0, (hipStream_t)stream, a);
        HIP_TRY(hipGetLastError());
    }
    return HAG_OK;
}

}  // extern "C"
