// The 2-norm of many tensors taken as one vector, and all of them scaled so that it is at most max_norm.
//   N = sqrt(sum of g^2),  c = N <= max_norm ? 1 : max_norm / N,  out = c g
#include "hag_elem.hpp"

#include <cmath>

namespace hag {

// The tensors are cut into units of at most `unit` elements, one workgroup each; a launch takes as many tensors as its argument block holds.
constexpr int kClipTensors = 112;
constexpr int64_t kClipUnits = 2048, kClipRound = 4096;
struct ClipArgs {
    struct Tensor {
        const void *in;
        void *out;
        int64_t count;
        int32_t dtype;
        int32_t first_unit;      // of this launch
    } t[kClipTensors];
    int64_t unit;
    int32_t tensors;
    int32_t units;               // of this launch
    int32_t partial_at;          // where this launch's units begin among those of all launches
    int32_t partials;            // units of all launches
};
static_assert(sizeof(ClipArgs) <= 3840, "kernel arguments are limited to 4 KB");

// the tensor of a unit: the last one that does not begin after it
__device__ __forceinline__ int clip_tensor(const ClipArgs &a, int unit) {
    int lo = 0, hi = a.tensors;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.t[mid].first_unit <= unit) lo = mid; else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ double block_sum64(double v, double *lds) {
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) v += __shfl_xor(v, off);
    if (threadIdx.x % kWave == 0) lds[threadIdx.x / kWave] = v;
    __syncthreads();
    v = 0.;
#pragma unroll
    for (int w = 0; w < kBlock / kWave; ++w) v += lds[w];
    return v;
}

// Pieces of a unit that a workgroup moves at a time: four vectors of 16 bytes for each thread, requested together.
constexpr int kClipAsk = 4;
template <typename T>
constexpr int kClipPiece = kClipAsk * kBlock * kVec<T>;

template <typename T>
__device__ __forceinline__ double sum_squares(const T *p, int64_t count) {
    constexpr int V = kVec<T>;
    double s[kClipAsk] = {};
    int64_t at = 0;
    for (; at + kClipPiece<T> <= count; at += kClipPiece<T>) {
        typename VecOf<T>::type raw[kClipAsk];
#pragma unroll
        for (int u = 0; u < kClipAsk; ++u) raw[u] = load_vec(p + at + (u * kBlock + threadIdx.x) * V);
#pragma unroll
        for (int u = 0; u < kClipAsk; ++u)
#pragma unroll
            for (int e = 0; e < V; ++e) { const double v = (double)(float)raw[u][e]; s[u] += v * v; }
    }
    for (int64_t i = at + threadIdx.x * V; i < count; i += kBlock * V) {
        const typename VecOf<T>::type raw = load_vec(p + i, i + V <= count, (int)min(count - i, (int64_t)V));
#pragma unroll
        for (int e = 0; e < V; ++e) { const double v = (double)(float)raw[e]; s[0] += v * v; }
    }
    return (s[0] + s[1]) + (s[2] + s[3]);
}

// Bound by reading: 30 M fp32 elements 22 us (5.4 TB/s).  Squares are taken and added up in 64 bits: the square of an fp32 gradient above 2e19 is no fp32 number.
__global__ __launch_bounds__(kBlock) void clip_sums_kernel(ClipArgs a, double *__restrict__ partial) {
    __shared__ double lds[kBlock / kWave];
    const int t = clip_tensor(a, blockIdx.x);
    const int64_t begin = (int64_t)(blockIdx.x - a.t[t].first_unit) * a.unit, count = min(a.unit, a.t[t].count - begin);
    const double s = a.t[t].dtype == HAG_F32    ? sum_squares((const float *)a.t[t].in + begin, count)
                     : a.t[t].dtype == HAG_BF16 ? sum_squares((const bf16_t *)a.t[t].in + begin, count)
                                                : sum_squares((const f16_t *)a.t[t].in + begin, count);
    const double sum = block_sum64(s, lds);
    if (threadIdx.x == 0) partial[a.partial_at + blockIdx.x] = sum;
}

// Last piece first: the end of every unit was read last and is still in the caches, where streaming stores leave it (30 M fp32 elements into other tensors 72 -> 59 us;
// with an update that reads them next 155 -> 148, but 4 M elements 26 -> 33: ordinary stores would leave those in the caches).
template <typename T>
__device__ __forceinline__ void scale_unit(const T *p, T *out, int64_t count, float c) {
    constexpr int V = kVec<T>;
    int64_t at = count / kClipPiece<T> * kClipPiece<T>;
    for (int64_t i = at + threadIdx.x * V; i < count; i += kBlock * V) {
        const int have = (int)min(count - i, (int64_t)V);
        const typename VecOf<T>::type raw = load_vec(p + i, have == V, have);
        float v[V];
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = (float)raw[e] * c;
        store_vec<true>(out + i, have, v);
    }
    while (at > 0) {
        at -= kClipPiece<T>;
        typename VecOf<T>::type raw[kClipAsk];
#pragma unroll
        for (int u = 0; u < kClipAsk; ++u) raw[u] = load_vec(p + at + (u * kBlock + threadIdx.x) * V);
#pragma unroll
        for (int u = 0; u < kClipAsk; ++u) {
            float v[V];
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = (float)raw[u][e] * c;
            store_vec<true>(out + at + (u * kBlock + threadIdx.x) * V, V, v);
        }
    }
}

// The same with a factor that is no fp32 number: rare, so without vectors in flight, whose registers the ordinary way would have to hold too (44 -> 71, bf16 32.3 -> 33.4 us).
template <typename T>
__device__ __forceinline__ void scale_unit_far(const T *p, T *out, int64_t count, double c) {
#pragma unroll 1
    for (int64_t i = threadIdx.x; i < count; i += kBlock) out[i] = (T)(float)((double)(float)p[i] * c);
}

// Bound by reading once more and writing: 30 M fp32 elements into other tensors 38 us (6.3 TB/s: part of what is read is still in the caches).  Every workgroup adds up all partial
// sums itself, in one order, rather than wait for one more launch.  What is left above one read and one write is the second read; tensors of this size would fit the
// registers and LDS of all compute units, but a wait of all workgroups for each other hangs where another stream holds some of their places.
__global__ __launch_bounds__(kBlock) void clip_scale_kernel(ClipArgs a, const double *__restrict__ partial, double max_norm, float *__restrict__ norm) {
    __shared__ double lds[kBlock / kWave];
    double s = 0.;
    for (int i = threadIdx.x; i < a.partials; i += 8 * kBlock) {
        double v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = partial[min(i + u * kBlock, a.partials - 1)];
#pragma unroll
        for (int u = 0; u < 8; ++u) s += i + u * kBlock < a.partials ? v[u] : 0.;
    }
    const double total = sqrt(block_sum64(s, lds));
    const double factor = total <= max_norm ? 1. : max_norm / total;       // (a NaN: NaN; an infinite norm: 0, and NaN for the infinite elements)
    const float c = (float)factor;
    if (blockIdx.x == 0 && a.partial_at == 0 && threadIdx.x == 0) *norm = (float)total;
    if ((int)blockIdx.x >= a.units) return;                // no element at all: the launch is there for the norm
    const int t = clip_tensor(a, blockIdx.x);
    if (c == 1.f && a.t[t].out == a.t[t].in) return;
    const int64_t begin = (int64_t)(blockIdx.x - a.t[t].first_unit) * a.unit, count = min(a.unit, a.t[t].count - begin);
    // A factor below 2^-126 has fewer bits in fp32, or none, where its products with gradients as large as their norm are ordinary numbers: those are taken in 64 bits.
    const bool far = c < 0x1p-126f;
    auto scale = [&](auto e) {
        using T = decltype(e);
        const T *in = (const T *)a.t[t].in + begin;
        T *out = (T *)a.t[t].out + begin;
        if (far) scale_unit_far(in, out, count, factor);
        else scale_unit(in, out, count, c);
    };
    if (a.t[t].dtype == HAG_F32) scale(float());
    else if (a.t[t].dtype == HAG_BF16) scale(bf16_t());
    else scale(f16_t());
}

}  // namespace hag

using namespace hag;

extern "C" {

// every tensor has at most one unit that is not full
size_t hag_clip_workspace_bytes(int64_t tensors) { return tensors < 0 || tensors > (1 << 24) ? 0 : (size_t)(kClipUnits + tensors) * sizeof(double); }

int hag_clip_gradients(int64_t tensors, const hag_tensor_t *list, double max_norm, float *norm, void *workspace, void *stream) {
    if (tensors < 0 || tensors > (1 << 24)) { set_error("number of tensors must be in 0 .. 2^24"); return HAG_EINVAL; }
    if (!(max_norm > 0.)) { set_error("max_norm must be positive"); return HAG_EINVAL; }
    if ((tensors > 0 && !list) || !norm || !workspace) { set_error("NULL pointer"); return HAG_EINVAL; }
    if ((uintptr_t)workspace & 15) { set_error("workspace must be 16-byte aligned"); return HAG_EINVAL; }
    int64_t total = 0;
    for (int64_t i = 0; i < tensors; ++i) {
        const hag_tensor_t &t = list[i];
        if (t.count < 0 || t.count > ((int64_t)1 << 48)) { set_error("count of a tensor out of range"); return HAG_EINVAL; }
        if (!elem_type((hag_dtype_t)t.dtype)) { set_error("elements are HAG_F32, HAG_BF16 or HAG_F16"); return HAG_EINVAL; }
        if (t.count > 0 && (!t.in || !t.out)) { set_error("NULL pointer"); return HAG_EINVAL; }
        total += t.count;
    }
    const int64_t unit = std::max<int64_t>(1, (total + kClipUnits * kClipRound - 1) / (kClipUnits * kClipRound)) * kClipRound;
    // the launches' argument blocks one after the other, first to add up, then to scale
    hipStream_t s = (hipStream_t)stream;
    int64_t partials = 0;
    for (int64_t i = 0; i < tensors; ++i) partials += (list[i].count + unit - 1) / unit;
    for (int pass = 0; pass < 2; ++pass) {
        int64_t at = 0, i = 0;
        do {
            ClipArgs a;
            a.unit = unit;
            a.tensors = a.units = 0;
            a.partial_at = (int32_t)at;
            a.partials = (int32_t)partials;
            for (; i < tensors && a.tensors < kClipTensors; ++i) {
                if (list[i].count == 0) continue;
                a.t[a.tensors++] = {list[i].in, list[i].out, list[i].count, list[i].dtype, a.units};
                a.units += (int32_t)((list[i].count + unit - 1) / unit);
            }
            if (pass == 0 && a.units > 0) hipLaunchKernelGGL(clip_sums_kernel, dim3((unsigned)a.units), dim3(kBlock), 0, s, a, (double *)workspace);
            if (pass == 1 && (a.units > 0 || at == 0))
                hipLaunchKernelGGL(clip_scale_kernel, dim3((unsigned)std::max(a.units, 1)), dim3(kBlock), 0, s, a, (const double *)workspace, max_norm, norm);
            HIP_TRY(hipGetLastError());
            at += a.units;
        } while (i < tensors);
    }
    return HAG_OK;
}

}  // extern "C"
