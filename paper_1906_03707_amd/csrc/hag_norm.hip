// Layer norm over the rows of a matrix, and its backward pass.
//   m = mean of x over a row, r = 1 / sqrt(mean of (x - m)^2 + eps), xh = (x - m) r, y = xh w + b
//   u = g_y w:  g_x = r (u - mean(u) - xh mean(u xh)),  g_w = sum over rows of g_y xh,  g_b = sum over rows of g_y
// A row is read once and stays in registers: LPR adjacent lanes hold K vectors of 16 bytes each (lane l vectors l, l + LPR, ...), sums over a row are moves
// between those lanes.  Statistics in fp32: a first mean m of the differences from the row's first element (rows of one value, however large, then have that
// mean and no deviation), then the sums of the deviations from it and of their squares.  The mean of the deviations is what m is off by: rounded to the grid of its own size (half of
// the spread for a row of 1e8 and 1e8 + 8), or by as much as the first element's grid where that stands out.  It is taken out of the mean, of the variance and of the deviations.
// Rows of more than 1024 columns take a workgroup, of more than 8192 are read again for every sum.
#include "hag_elem.hpp"

namespace hag {

struct NormArgs {
    const void *x, *gy;
    int64_t x_stride, gy_stride, n;
    int64_t x_extent, gy_extent;     // elements from the first of the matrix to the end of its last row: what may be read
    int32_t d, param32;              // param32: weight and bias are fp32, else they have the type of x
    const void *weight, *bias;       // or NULL
    float eps, inv_d;
    void *out;                       // y or g_x, contiguous
    const float *mean_in, *rstd_in;
    float *mean, *rstd;              // or NULL
    float *partial;                  // g_w and g_b of every workgroup [groups, 2, d]; NULL: not wanted, or one workgroup does it all
    void *g_w, *g_b;                 // for one workgroup
};

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

// Rows of finite numbers whose differences or squares add up beyond fp32 are taken again times 2^-80: below 2^48 then, squares of differences of 2^20 columns add up to less
// than 2^118.  Some deviation was 2^54 or more, so what is lost below 2^-149 is nothing beside the spread.  (fp16 numbers cannot get there.)
constexpr float kFarScale = 0x1p-80f;
template <typename T>
constexpr bool kFarRows = !std::is_same<T, f16_t>::value;

// mean of the squares of (deviations - off), off their mean; NaN stays
__device__ __forceinline__ float variance(float squares, float off) {
    const float v = fmaf(-off, off, squares);
    return v < 0.f ? 0.f : v;
}

// (x - m) r by halves: the difference of two fp32 numbers may be no fp32 number, that of their halves is one
__device__ __forceinline__ float normed(float x, float m, float r) { return fmaf(x, 0.5f, -0.5f * m) * (2.f * r); }

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

// A row beyond fp32 (`here`; other rows' lanes go along), read again for every sum: rows that nothing but a broken training meets, so what counts is that the ordinary ones do not
// hold registers for them.
template <typename T, int LPR>
__device__ __forceinline__ void norm_far_row(const NormArgs &a, int64_t row, bool here, float2 (*lds)[16], int &turn) {
    const int l = threadIdx.x % LPR;
    const T *p = (const T *)a.x + min(row, a.n - 1) * a.x_stride;
    const float first = (float)p[0] * kFarScale;
    float2 s = make_float2(0.f, 0.f);
#pragma unroll 1
    for (int c = l; c < a.d; c += LPR) s.x += (float)p[c] * kFarScale - first;
    const float m = first + row_sums<LPR>(s, lds, turn).x * a.inv_d;
    s.x = 0.f;
#pragma unroll 1
    for (int c = l; c < a.d; c += LPR) {
        const float v = (float)p[c] * kFarScale - m;
        s.x += v * v;
        s.y += v;
    }
    s = row_sums<LPR>(s, lds, turn);
    const float off = s.y * a.inv_d, r = inverse_root(variance(s.x * a.inv_d, off) + a.eps * kFarScale * kFarScale);
    if (!here) return;
#pragma unroll 1
    for (int c = l; c < a.d; c += LPR) {
        const float xh = ((float)p[c] * kFarScale - m - off) * r;
        ((T *)a.out)[row * a.d + c] = (T)(xh * (a.weight ? param(a.weight, a.param32, T(), c) : 1.f) + (a.bias ? param(a.bias, a.param32, T(), c) : 0.f));
    }
    if (l == 0) {
        if (a.mean) a.mean[row] = (m + off) / kFarScale;
        if (a.rstd) a.rstd[row] = r * kFarScale;
    }
}

// Bound by reading x and writing y.  Every lane requests R rows one after the other before it needs the first.  232965 x 128 fp32 40.5 us, bf16 21.2 (5.9 and 5.7 TB/s; a copy: 5.3).
// 56944 x 251 bf16 15.2 us, x 256 12.1: the same bytes from and to memory, but 1.4 times the vector instructions (which columns count) and twice the stores (rows' ends, element by element).
template <typename T, int LPR, int K, int R, bool TAIL>
__global__ __launch_bounds__(kNormBlock<LPR>) void norm_kernel(NormArgs a) {
    __shared__ float2 lds[2][16];
    typedef typename VecOf<T>::type Raw;
    constexpr int V = kVec<T>, kTaker = LPR <= kWave ? kWave : LPR;
    const int l = threadIdx.x % LPR;
    const int64_t row0 = ((int64_t)blockIdx.x * (kNormBlock<LPR> / kTaker) + threadIdx.x / kTaker) * (kSide<LPR> * R) + threadIdx.x % kTaker / LPR;
    const T *x = (const T *)a.x;
    float v[R][K][V], first[R], m[R], off[R], r[R];
    uint32_t far = 0;                                      // bits of rows beyond fp32
    int turn = 0;
    {
        Raw raw[R][K];
#pragma unroll
        for (int t = 0; t < R; ++t) {
            const int64_t at = min(row0 + t * kSide<LPR>, a.n - 1) * a.x_stride;   // (rows beyond the last one: that one again, not stored)
            first[t] = (float)x[at];
#pragma unroll
            for (int k = 0; k < K; ++k) raw[t][k] = load_columns<T, TAIL>(x, at, (l + LPR * k) * V, a.d, a.x_extent);
        }
#pragma unroll
        for (int t = 0; t < R; ++t)
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int e = 0; e < V; ++e) v[t][k][e] = (float)raw[t][k][e];
    }
#pragma unroll
    for (int t = 0; t < R; ++t) {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int col = (l + LPR * k) * V;
            float part = 0.f;
#pragma unroll
            for (int e = 0; e < V; ++e) part += !TAIL || col + e < a.d ? v[t][k][e] - first[t] : 0.f;
            s += col < a.d ? part : 0.f;
        }
        m[t] = first[t] + row_sums<LPR>(make_float2(s, 0.f), lds, turn).x * a.inv_d;
        float2 q = make_float2(0.f, 0.f);                  // squares of the deviations, deviations
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int col = (l + LPR * k) * V;
            float2 part = make_float2(0.f, 0.f);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                v[t][k][e] -= m[t];
                part.x += !TAIL || col + e < a.d ? v[t][k][e] * v[t][k][e] : 0.f;
                part.y += !TAIL || col + e < a.d ? v[t][k][e] : 0.f;
            }
            q.x += col < a.d ? part.x : 0.f;
            q.y += col < a.d ? part.y : 0.f;
        }
        q = row_sums<LPR>(q, lds, turn);
        off[t] = q.y * a.inv_d;
        m[t] += off[t];
        r[t] = inverse_root(variance(q.x * a.inv_d, off[t]) + a.eps);
        if (kFarRows<T> && !(q.x < INFINITY) && row0 + t * kSide<LPR> < a.n) far |= 1u << t;
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int col = (l + LPR * k) * V;
        if (col >= a.d) continue;
        float w[V], b[V];
        load_params<T, TAIL>(a.weight, a.param32, col, a.d, 1.f, w);
        load_params<T, TAIL>(a.bias, a.param32, col, a.d, 0.f, b);
#pragma unroll
        for (int t = 0; t < R; ++t) {
            const int64_t row = row0 + t * kSide<LPR>;
            if (row >= a.n || far >> t & 1) continue;
#pragma unroll
            for (int e = 0; e < V; ++e) v[t][k][e] = (v[t][k][e] - off[t]) * r[t] * w[e] + b[e];
            store_vec((T *)a.out + row * a.d + col, TAIL ? a.d - col : V, v[t][k]);
        }
    }
#pragma unroll
    for (int t = 0; t < R; ++t) {
        const int64_t row = row0 + t * kSide<LPR>;
        if (l == 0 && row < a.n && !(far >> t & 1)) {
            if (a.mean) a.mean[row] = m[t];
            if (a.rstd) a.rstd[row] = r[t];
        }
    }
    if (kFarRows<T> && __any(far != 0)) {                  // (a row of more than a wavefront: the same in all of them)
#pragma unroll 1
        for (int t = 0; t < R; ++t) norm_far_row<T, LPR>(a, row0 + t * kSide<LPR>, far >> t & 1, lds, turn);
    }
}

// Bound by reading x and g_y and writing g_x.  Workgroups take rows in turn, keep the sums of their columns for g_w and g_b in registers, and leave them in `partial`, one
// row of 2 d for each workgroup, added up in a fixed order by norm_reduce_kernel.  The next rows are requested before the present ones are worked on.
// 65536 x 512 fp32 78 us with the last sums (5.2 TB/s), 232965 x 128 bf16 35 (5.1), 56944 x 251 bf16 21 (4.1).
template <typename T, int LPR, int K, int R, bool TAIL>
__global__ __launch_bounds__(kGradBlock<LPR>) void norm_grad_kernel(NormArgs a) {
    extern __shared__ float sums[];                        // [wavefronts][2][LPR * K * V], rows of up to 64 lanes
    __shared__ float2 lds[2][16];
    typedef typename VecOf<T>::type Raw;
    constexpr int V = kVec<T>, kTaker = LPR <= kWave ? kWave : LPR, kTakers = kGradBlock<LPR> / kTaker;   // what takes a set of rows: a wavefront, or the workgroup
    const int l = threadIdx.x % LPR, side = threadIdx.x % kTaker / LPR;
    const T *x = (const T *)a.x, *gy = (const T *)a.gy;
    int turn = 0;
    float w[K][V], gw[K][V], gb[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        load_params<T, TAIL>(a.weight, a.param32, (l + LPR * k) * V, a.d, 1.f, w[k]);
#pragma unroll
        for (int e = 0; e < V; ++e) gw[k][e] = gb[k][e] = 0.f;
    }
    const int64_t sets = (a.n + kSide<LPR> * R - 1) / (kSide<LPR> * R), step = (int64_t)gridDim.x * kTakers;
    struct Rows {
        Raw x[R][K], g[R][K];
        float m[R], r[R];
    };
    auto request = [&](int64_t set, Rows &q) {
#pragma unroll
        for (int t = 0; t < R; ++t) {
            const int64_t row = min((set * R + t) * kSide<LPR> + side, a.n - 1);
            q.m[t] = a.mean_in[row];
            q.r[t] = a.rstd_in[row];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                q.x[t][k] = load_columns<T, TAIL>(x, row * a.x_stride, (l + LPR * k) * V, a.d, a.x_extent);
                q.g[t][k] = load_columns<T, TAIL>(gy, row * a.gy_stride, (l + LPR * k) * V, a.d, a.gy_extent);
            }
        }
    };
    auto work = [&](int64_t set, const Rows &q) {
#pragma unroll
        for (int t = 0; t < R; ++t) {
            const int64_t row = (set * R + t) * kSide<LPR> + side;
            const bool here = row < a.n;
            float2 s = make_float2(0.f, 0.f);
            float xh[K][V], u[K][V];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int col = (l + LPR * k) * V;
                float2 part = make_float2(0.f, 0.f);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const bool in = here && (!TAIL || col + e < a.d);
                    const float g = in ? (float)q.g[t][k][e] : 0.f;
                    xh[k][e] = in ? normed((float)q.x[t][k][e], q.m[t], q.r[t]) : 0.f;
                    u[k][e] = g * w[k][e];
                    gw[k][e] += g * xh[k][e];              // (columns beyond the row's end: not read)
                    gb[k][e] += g;
                    part.x += u[k][e];
                    part.y += u[k][e] * xh[k][e];
                }
                s.x += col < a.d ? part.x : 0.f;
                s.y += col < a.d ? part.y : 0.f;
            }
            s = row_sums<LPR>(s, lds, turn);
            s.x *= a.inv_d;
            s.y *= a.inv_d;
            if (!here) continue;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int col = (l + LPR * k) * V;
                if (col >= a.d) continue;
#pragma unroll
                for (int e = 0; e < V; ++e) u[k][e] = q.r[t] * (u[k][e] - s.x - xh[k][e] * s.y);
                store_vec((T *)a.out + row * a.d + col, TAIL ? a.d - col : V, u[k]);
            }
        }
    };
    int64_t set = (int64_t)blockIdx.x * kTakers + threadIdx.x / kTaker;
    if (set < sets) {
        Rows q;
        request(set, q);
        for (; set < sets; set += step) {
            Rows next = q;
            if (set + step < sets) request(set + step, next);
            work(set, q);
            q = next;
        }
    }
    if (!a.partial && !a.g_w && !a.g_b) return;
    auto leave = [&](int c, float w_sum, float b_sum) {
        if (a.partial) {
            a.partial[(int64_t)blockIdx.x * 2 * a.d + c] = w_sum;
            a.partial[((int64_t)blockIdx.x * 2 + 1) * a.d + c] = b_sum;
        } else if (a.param32) {
            if (a.g_w) ((float *)a.g_w)[c] = w_sum;
            if (a.g_b) ((float *)a.g_b)[c] = b_sum;
        } else {
            if (a.g_w) ((T *)a.g_w)[c] = (T)w_sum;
            if (a.g_b) ((T *)a.g_b)[c] = (T)b_sum;
        }
    };
    if (LPR > kWave) {                                     // every column has one lane
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int e = 0; e < V; ++e)
                if ((l + LPR * k) * V + e < a.d) leave((l + LPR * k) * V + e, gw[k][e], gb[k][e]);
        return;
    }
    // lanes that hold the same columns, then the wavefronts in their order
    constexpr int kWidth = LPR * K * V;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e)
#pragma unroll
            for (int off = LPR; off < kWave; off <<= 1) {
                gw[k][e] += __shfl_xor(gw[k][e], off);
                gb[k][e] += __shfl_xor(gb[k][e], off);
            }
    if (threadIdx.x % kWave < LPR) {
        float *mine = sums + threadIdx.x / kWave * (2 * kWidth);
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                mine[(l + LPR * k) * V + e] = gw[k][e];
                mine[kWidth + (l + LPR * k) * V + e] = gb[k][e];
            }
    }
    __syncthreads();
    for (int c = threadIdx.x; c < a.d; c += kGradBlock<LPR>) {
        float w_sum = 0.f, b_sum = 0.f;
#pragma unroll
        for (int wave = 0; wave < kTakers; ++wave) {
            w_sum += sums[wave * 2 * kWidth + c];
            b_sum += sums[(wave * 2 + 1) * kWidth + c];
        }
        leave(c, w_sum, b_sum);
    }
}

// g_w and g_b: 16 columns per workgroup, 64 threads for each, which take every 64th row of `partial`, then those in a fixed order
template <typename P>
__global__ __launch_bounds__(1024) void norm_reduce_kernel(const float *__restrict__ partial, int32_t groups, int32_t d, P *__restrict__ g_w, P *__restrict__ g_b) {
    __shared__ float part[64][17];
    const int o = threadIdx.x & 15, p = threadIdx.x >> 4, i = blockIdx.x * 16 + o;
    float sum = 0.f;
    if (i < 2 * d) {
#pragma unroll 8
        for (int g = p; g < groups; g += 64) sum += partial[(int64_t)g * 2 * d + i];
    }
    part[p][o] = sum;
    __syncthreads();
    for (int half = 32; half > 0; half >>= 1) {
        if (p < half) part[p][o] += part[p + half][o];
        __syncthreads();
    }
    if (p != 0 || i >= 2 * d) return;
    if (i < d) {
        if (g_w) g_w[i] = (P)part[0][o];
    } else if (g_b) {
        g_b[i - d] = (P)part[0][o];
    }
}

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

template <typename T>
__global__ __launch_bounds__(kWide) void norm_wide_kernel(NormArgs a) {
    __shared__ float2 lds[kWide / kWave];
    const int64_t row = blockIdx.x;
    const T *p = (const T *)a.x + row * a.x_stride;
    float scale = 1.f, m, off, r;
    for (;;) {                                             // (once, for rows beyond fp32 twice)
        const float first = (float)p[0] * scale;
        float2 s = make_float2(0.f, 0.f);
        for (int c = threadIdx.x; c < a.d; c += kWide) s.x += (float)p[c] * scale - first;
        m = first + wide_sums(s, lds).x * a.inv_d;
        s.x = 0.f;
        for (int c = threadIdx.x; c < a.d; c += kWide) {
            const float v = (float)p[c] * scale - m;
            s.x += v * v;
            s.y += v;
        }
        s = wide_sums(s, lds);
        off = s.y * a.inv_d;
        r = inverse_root(variance(s.x * a.inv_d, off) + a.eps * scale * scale);
        if (!kFarRows<T> || scale != 1.f || s.x < INFINITY) break;
        scale = kFarScale;
    }
    for (int c = threadIdx.x; c < a.d; c += kWide) {
        const float xh = ((float)p[c] * scale - m - off) * r;
        ((T *)a.out)[row * a.d + c] = (T)(xh * (a.weight ? param(a.weight, a.param32, T(), c) : 1.f) + (a.bias ? param(a.bias, a.param32, T(), c) : 0.f));
    }
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[row] = (m + off) / scale;
        if (a.rstd) a.rstd[row] = r * scale;
    }
}

template <typename T>
__global__ __launch_bounds__(kWide) void norm_grad_wide_kernel(NormArgs a) {
    __shared__ float2 lds[kWide / kWave];
    const int64_t row = blockIdx.x;
    const T *p = (const T *)a.x + row * a.x_stride, *g = (const T *)a.gy + row * a.gy_stride;
    const float m = a.mean_in[row], r = a.rstd_in[row];
    float2 s = make_float2(0.f, 0.f);
    for (int c = threadIdx.x; c < a.d; c += kWide) {
        const float u = (float)g[c] * (a.weight ? param(a.weight, a.param32, T(), c) : 1.f);
        s.x += u;
        s.y += u * normed((float)p[c], m, r);
    }
    s = wide_sums(s, lds);
    const float s1 = s.x * a.inv_d, s2 = s.y * a.inv_d;
    for (int c = threadIdx.x; c < a.d; c += kWide) {
        const float u = (float)g[c] * (a.weight ? param(a.weight, a.param32, T(), c) : 1.f);
        ((T *)a.out)[row * a.d + c] = (T)(r * (u - s1 - normed((float)p[c], m, r) * s2));
    }
}

// partial[slice] = the sums of a slice of the rows, 64 columns per workgroup
template <typename T>
__global__ __launch_bounds__(kBlock) void norm_wide_sums_kernel(NormArgs a) {
    __shared__ float lds[kBlock / kWave][2][kWave];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, c = blockIdx.x * kWave + lane;
    float gw = 0.f, gb = 0.f;
    if (c < a.d) {
        for (int64_t row = (int64_t)blockIdx.y * (kBlock / kWave) + wave; row < a.n; row += (int64_t)gridDim.y * (kBlock / kWave)) {
            const float g = (float)((const T *)a.gy)[row * a.gy_stride + c];
            gw += g * normed((float)((const T *)a.x)[row * a.x_stride + c], a.mean_in[row], a.rstd_in[row]);
            gb += g;
        }
    }
    lds[wave][0][lane] = gw;
    lds[wave][1][lane] = gb;
    __syncthreads();
    if (wave > 0 || c >= a.d) return;
    for (int v = 1; v < kBlock / kWave; ++v) { gw += lds[v][0][lane]; gb += lds[v][1][lane]; }
    a.partial[((int64_t)blockIdx.y * 2) * a.d + c] = gw;
    a.partial[((int64_t)blockIdx.y * 2 + 1) * a.d + c] = gb;
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

typedef void (*norm_kernel_t)(NormArgs);
// Workgroups that take `rows` rows each, whatever a launch holds.
template <typename T>
static int launch_rows(norm_kernel_t kernel, const NormArgs &a, int64_t rows, int threads, hipStream_t s) {
    return launch_parts((a.n + rows - 1) / rows, threads, [&](int64_t first, int64_t count) {
        const int64_t at = first * rows;
        NormArgs part = a;
        part.n = std::min(count * rows, a.n - at);
        part.x = (const T *)a.x + at * a.x_stride;
        part.x_extent = (part.n - 1) * a.x_stride + a.d;
        part.gy = a.gy ? (const T *)a.gy + at * a.gy_stride : nullptr;
        part.gy_extent = (part.n - 1) * a.gy_stride + a.d;
        part.out = (T *)a.out + at * a.d;
        part.mean_in = a.mean_in ? a.mean_in + at : nullptr;
        part.rstd_in = a.rstd_in ? a.rstd_in + at : nullptr;
        part.mean = a.mean ? a.mean + at : nullptr;
        part.rstd = a.rstd ? a.rstd + at : nullptr;
        hipLaunchKernelGGL(kernel, dim3((unsigned)count), dim3((unsigned)threads), 0, s, part);
    });
}
template <typename T, template <int, int> class F>
static norm_kernel_t norm_pick(NormShape s) {
    switch (s.lpr) {
    case 2: return F<2, 1>::kernel;
    case 4: return F<4, 1>::kernel;
    case 8: return F<8, 1>::kernel;
    case 16: return F<16, 1>::kernel;
    case 32: return F<32, 1>::kernel;
    case 64:
        if constexpr (kVec<T> == 4) {
            if (s.k > 2) return s.k == 3 ? (norm_kernel_t)F<64, 3>::kernel : (norm_kernel_t)F<64, 4>::kernel;
        }
        return s.k == 1 ? (norm_kernel_t)F<64, 1>::kernel : (norm_kernel_t)F<64, 2>::kernel;
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
// Rows one after the other that a lane requests at once.  Forward: 16 columns' worth, against 8: 65536 x 512 fp32 43.5 us and 45.4, 232965 x 128 bf16 21.3 and 22.0, 56944 x 251 bf16 15.3
// and 17.3, but 232965 x 128 fp32 40.4 and 39.7, 370000 x 64 fp32 34.0 and 33.2.
constexpr int norm_rows(int lpr, int k, int vec) { return lpr > kWave || k * vec >= 16 ? 1 : 16 / (k * vec); }
constexpr int norm_grad_rows(int lpr, int k) { return lpr <= kWave && k == 1 ? 2 : 1; }
// Threads of a workgroup, and the rows that it takes side by side.
static int norm_block(NormShape s, bool backward) { return s.lpr <= kWave ? (backward ? 2 * kBlock : kBlock) : s.lpr; }
static int64_t norm_side(NormShape s, bool backward) { return norm_block(s, backward) / s.lpr; }
template <typename T, bool TAIL>
struct Forward {
    template <int LPR, int K>
    struct Of { static constexpr auto kernel = norm_kernel<T, LPR, K, norm_rows(LPR, K, kVec<T>), TAIL>; };
};
template <typename T, bool TAIL>
struct Backward {
    template <int LPR, int K>
    struct Of { static constexpr auto kernel = norm_grad_kernel<T, LPR, K, norm_grad_rows(LPR, K), TAIL>; };
};

// Workgroups of a backward pass.  One for each of the 256 compute units, so that few partial sums are written and read again; two where rows are shorter than a wavefront and those
// sums are small (370000 x 64 fp32: 52.9 us with 256, 51.9 with 512; 65536 x 512 79.9 and 81.5, 16384 x 1024 38.8 and 41.2).
constexpr int64_t kNormSlices = 128;
static int64_t norm_grad_groups(int64_t n, NormShape s) {
    if (s.k == 0) return kNormSlices;
    const int64_t rows = s.lpr <= kWave ? norm_side(s, true) * norm_grad_rows(s.lpr, s.k) * 4 : 8;
    return std::max<int64_t>(1, std::min<int64_t>((n + rows - 1) / rows, s.lpr < kWave ? 512 : 256));
}

}  // namespace hag

using namespace hag;

extern "C" {

static const char *norm_refusal(int64_t n, int64_t d, hag_dtype_t dtype, hag_dtype_t param_dtype) {
    if (n < 0 || d <= 0 || n > 0x7fffffffLL || d > (1 << 20)) return "n must be in 0 .. 2^31 - 1, d in 1 .. 2^20";
    if (!elem_type(dtype)) return "elements are HAG_F32, HAG_BF16 or HAG_F16";
    if (param_dtype != dtype && param_dtype != HAG_F32) return "weight and bias have the elements' type or HAG_F32";
    return nullptr;
}

int hag_layer_norm(int64_t n, int64_t d, hag_dtype_t dtype, const void *x, int64_t x_stride, hag_dtype_t param_dtype, const void *weight, const void *bias, float eps, void *y,
                   float *mean, float *rstd, void *stream) {
    if (const char *why = norm_refusal(n, d, dtype, param_dtype)) { set_error(why); return HAG_EINVAL; }
    if (x_stride < 0) { set_error("negative row stride"); return HAG_EINVAL; }
    if (!(eps >= 0.f)) { set_error("eps must not be negative"); return HAG_EINVAL; }
    if (n == 0) return HAG_OK;
    if (!x || !y) { set_error("NULL pointer"); return HAG_EINVAL; }
    NormArgs a = {};
    a.x = x;
    a.x_stride = x_stride;
    a.n = n;
    a.x_extent = (n - 1) * x_stride + d;
    a.d = (int32_t)d;
    a.param32 = param_dtype == HAG_F32;
    a.weight = weight;
    a.bias = bias;
    a.eps = eps;
    a.inv_d = 1.f / (float)d;
    a.out = y;
    a.mean = mean;
    a.rstd = rstd;
    return elem_switch(dtype, [&](auto e) {
        using T = decltype(e);
        const NormShape s = norm_shape(d, kVec<T>);
        if (s.k == 0) return launch_rows<T>(norm_wide_kernel<T>, a, 1, kWide, (hipStream_t)stream);
        const norm_kernel_t kernel = d % kVec<T> ? norm_pick<T, Forward<T, true>::template Of>(s) : norm_pick<T, Forward<T, false>::template Of>(s);
        return launch_rows<T>(kernel, a, norm_side(s, false) * norm_rows(s.lpr, s.k, kVec<T>), norm_block(s, false), (hipStream_t)stream);
    });
}

size_t hag_layer_norm_grad_workspace_bytes(int64_t n, int64_t d) {
    if (norm_refusal(n, d, HAG_F32, HAG_F32)) return 0;
    // the types of 16 bits take fewer lanes to a row and no more workgroups
    return (size_t)std::max(norm_grad_groups(n, norm_shape(d, 4)), norm_grad_groups(n, norm_shape(d, 8))) * 2 * (size_t)d * sizeof(float);
}

int hag_layer_norm_grad(int64_t n, int64_t d, hag_dtype_t dtype, const void *g_y, int64_t g_y_stride, const void *x, int64_t x_stride, hag_dtype_t param_dtype, const void *weight,
                        const float *mean, const float *rstd, void *g_x, void *g_weight, void *g_bias, void *workspace, void *stream) {
    if (const char *why = norm_refusal(n, d, dtype, param_dtype)) { set_error(why); return HAG_EINVAL; }
    if (x_stride < 0 || g_y_stride < 0) { set_error("negative row stride"); return HAG_EINVAL; }
    const bool params = g_weight || g_bias;
    if ((n > 0 && (!g_y || !x || !mean || !rstd || !g_x)) || (params && !workspace)) { set_error("NULL pointer"); return HAG_EINVAL; }
    if ((uintptr_t)workspace & 15) { set_error("workspace must be 16-byte aligned"); return HAG_EINVAL; }
    if (n == 0 && !params) return HAG_OK;
    hipStream_t s = (hipStream_t)stream;
    NormArgs a = {};
    a.x = x;
    a.gy = g_y;
    a.x_stride = x_stride;
    a.gy_stride = g_y_stride;
    a.n = n;
    a.x_extent = n > 0 ? (n - 1) * x_stride + d : 0;
    a.gy_extent = n > 0 ? (n - 1) * g_y_stride + d : 0;
    a.d = (int32_t)d;
    a.param32 = param_dtype == HAG_F32;
    a.weight = weight;
    a.inv_d = 1.f / (float)d;
    a.out = g_x;
    a.mean_in = mean;
    a.rstd_in = rstd;
    return elem_switch(dtype, [&](auto e) {
        using T = decltype(e);
        const NormShape shape = norm_shape(d, kVec<T>);
        const int64_t groups = norm_grad_groups(n, shape);
        if (groups > 1) {
            a.partial = params ? (float *)workspace : nullptr;
        } else {
            a.g_w = g_weight;
            a.g_b = g_bias;
        }
        if (shape.k == 0) {
            if (const int rc = launch_rows<T>(norm_grad_wide_kernel<T>, a, 1, kWide, s)) return rc;
            if (params) hipLaunchKernelGGL(norm_wide_sums_kernel<T>, dim3((unsigned)((d + kWave - 1) / kWave), (unsigned)groups), dim3(kBlock), 0, s, a);
        } else {
            const size_t lds = shape.lpr <= kWave ? (size_t)(norm_block(shape, true) / kWave) * shape.lpr * shape.k * kVec<T> * 2 * sizeof(float) : 0;
            const norm_kernel_t kernel = d % kVec<T> ? norm_pick<T, Backward<T, true>::template Of>(shape) : norm_pick<T, Backward<T, false>::template Of>(shape);
            hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3((unsigned)norm_block(shape, true)), lds, s, a);
        }
        HIP_TRY(hipGetLastError());
        if (!a.partial) return (int)HAG_OK;
        const dim3 grid((unsigned)((2 * d + 15) / 16)), block(1024);
        if (a.param32) hipLaunchKernelGGL(norm_reduce_kernel<float>, grid, block, 0, s, a.partial, (int32_t)groups, (int32_t)d, (float *)g_weight, (float *)g_bias);
        else hipLaunchKernelGGL(norm_reduce_kernel<T>, grid, block, 0, s, a.partial, (int32_t)groups, (int32_t)d, (T *)g_weight, (T *)g_bias);
        HIP_TRY(hipGetLastError());
        return (int)HAG_OK;
    });
}

}  // extern "C"
