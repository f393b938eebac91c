// What layer norm and root-mean-square norm share: how a row is held in registers, its parameters, sums over its lanes.
#pragma once
#include "hag_elem.hpp"

namespace hag {

// weight or bias of the columns of a vector; `otherwise` where there is none
template <typename T, bool TAIL>
__device__ __forceinline__ void load_params(const void *p, int param32, int col, int d, float otherwise, float (&v)[kVec<T>]) {
#pragma unroll
    for (int e = 0; e < kVec<T>; ++e) v[e] = otherwise;
    if (!p || col >= d) return;
    if (!param32) {
        const typename VecOf<T>::type raw = load_vec((const T *)p + col, !TAIL || col + kVec<T> <= d, d - col);
#pragma unroll
        for (int e = 0; e < kVec<T>; ++e) v[e] = (float)raw[e];
        return;
    }
#pragma unroll
    for (int q = 0; q < kVec<T>; q += 4) {
        const typename VecOf<float>::type raw = load_vec((const float *)p + col + q, !TAIL || col + q + 4 <= d, d - col - q);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[q + e] = raw[e];
    }
}

// Sums over a row, in all of its lanes.  Rows of up to 64 lanes: moves between lanes; longer ones: the workgroup, through LDS (two halves, used in turn, so that one barrier
// a sum is enough).
template <int LPR>
__device__ __forceinline__ float2 row_sums(float2 v, float2 (*lds)[16], int &turn) {
    v.x = lanes_sum<(LPR <= kWave ? LPR : kWave)>(v.x);
    v.y = lanes_sum<(LPR <= kWave ? LPR : kWave)>(v.y);
    if (LPR <= kWave) return v;
    if (threadIdx.x % kWave == 0) lds[turn][threadIdx.x / kWave] = v;
    __syncthreads();
    v = make_float2(0.f, 0.f);
#pragma unroll
    for (int w = 0; w < LPR / kWave; ++w) {
        v.x += lds[turn][w].x;
        v.y += lds[turn][w].y;
    }
    turn ^= 1;
    return v;
}

// 1 / sqrt(v): the hardware's (one unit in the last place), and one step of Newton's method (half of one)
__device__ __forceinline__ float inverse_root(float v) {
    const float r = rsqrtf(v), better = fmaf(0.5f * r, fmaf(-(v * r), r, 1.f), r);
    return r > 0.f && r < INFINITY ? better : r;           // (v infinite, zero or no number: as it is)
}

// Element types whose squares may be beyond fp32.
template <typename T>
constexpr bool kFarRows = !std::is_same<T, f16_t>::value;

__device__ __forceinline__ float param(const void *p, int param32, float, int c) { return ((const float *)p)[c]; }
template <typename T>
__device__ __forceinline__ float param(const void *p, int param32, T, int c) { return param32 ? ((const float *)p)[c] : (float)((const T *)p)[c]; }

// Threads of a workgroup whose rows have LPR lanes (backward: twice as many where rows have a wavefront or less, so that there are half as many partial sums), and the rows
// that a wavefront (or the workgroup) takes side by side.
template <int LPR>
constexpr int kNormBlock = LPR <= kWave ? kBlock : LPR;
template <int LPR>
constexpr int kGradBlock = LPR <= kWave ? 2 * kBlock : LPR;
template <int LPR>
constexpr int kSide = LPR <= kWave ? kWave / LPR : 1;

// Rows that registers do not hold: a workgroup of 1024 reads its row again for every sum.
constexpr int kWide = 1024;
__device__ __forceinline__ float2 wide_sums(float2 v, float2 *lds) {
    v.x = lanes_sum<kWave>(v.x);
    v.y = lanes_sum<kWave>(v.y);
    __syncthreads();
    if (threadIdx.x % kWave == 0) lds[threadIdx.x / kWave] = v;
    __syncthreads();
    v = make_float2(0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kWide / kWave; ++w) {
        v.x += lds[w].x;
        v.y += lds[w].y;
    }
    return v;
}

// How a row is held: lanes per row, vectors per lane (0: not in registers).  A lane has at most 16 columns, whose gradients of weight and bias take as many registers each.
struct NormShape { int lpr, k; };
static NormShape norm_shape(int64_t d, int vec) {
    const int64_t nv = (d + vec - 1) / vec;
    int lpr = 2;
    while (lpr < kWave && lpr < nv) lpr *= 2;
    if (nv <= (16 / vec) * kWave) return {lpr, (int)((nv + kWave - 1) / kWave)};
    if (nv <= 256) return {256, 1};
    return nv <= 512 ? NormShape{256, 2} : nv <= 1024 ? NormShape{1024, 1} : nv <= 2048 && vec == 4 ? NormShape{1024, 2} : NormShape{1024, 0};
}

// The kernel of a shape: F<lanes, vectors>::kernel, of the pointer type P.
template <typename P, typename T, template <int, int> class F>
static P norm_pick(NormShape s) {
    switch (s.lpr) {
    case 2: return F<2, 1>::kernel;
    case 4: return F<4, 1>::kernel;
    case 8: return F<8, 1>::kernel;
    case 16: return F<16, 1>::kernel;
    case 32: return F<32, 1>::kernel;
    case 64:
        if constexpr (kVec<T> == 4) {
            if (s.k > 2) return s.k == 3 ? (P)F<64, 3>::kernel : (P)F<64, 4>::kernel;
        }
        return s.k == 1 ? (P)F<64, 1>::kernel : (P)F<64, 2>::kernel;
    case 256:
        if constexpr (kVec<T> == 8) {
            if (s.k == 1) return F<256, 1>::kernel;
        }
        return F<256, 2>::kernel;
    default:
        if constexpr (kVec<T> == 4) {
            if (s.k == 2) return F<1024, 2>::kernel;
        }
        return F<1024, 1>::kernel;
    }
}
// Threads of a workgroup, and the rows that it takes side by side.
static int norm_block(NormShape s, bool backward) { return s.lpr <= kWave ? (backward ? 2 * kBlock : kBlock) : s.lpr; }
static int64_t norm_side(NormShape s, bool backward) { return norm_block(s, backward) / s.lpr; }

}  // namespace hag
