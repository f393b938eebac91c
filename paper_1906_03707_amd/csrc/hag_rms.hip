// Root-mean-square norm over the rows of a matrix with the residual's addition, its output in the rows' type or in 8 bits, and its backward pass.
//   h = x + residual, rounded to the rows' type: what is kept is what is normed, so that the backward pass sees the same numbers
//   r = 1 / sqrt(mean of h^2 + eps), y = h r w
//   u = g_y w, xh = h r:  g_x = g_residual = r (u - xh mean(u xh)) + g_h,  g_w = sum over rows of g_y xh
// A row is read once and stays in registers, as in layer norm: LPR adjacent lanes hold K vectors of 16 bytes each.  Squares are added up in fp32, those of a lane first.
// Rows of more than 1024 columns take a workgroup, of more than 8192 are read again.
#include "hag_fp8.hpp"
#include "hag_norm_common.hpp"

namespace hag {

struct RmsArgs {
    const void *x, *res;             // res: the residual, or NULL
    int64_t x_stride, res_stride, n;
    int64_t x_extent, res_extent;    // elements from the first of the matrix to the end of its last row: what may be read
    int32_t d, param32;              // param32: weight is fp32, else it has the type of x
    const void *weight;              // or NULL
    float eps, inv_d;
    void *h;                         // x + residual, contiguous; NULL without a residual
    void *y;                         // contiguous
    float *rstd;                     // or NULL
    uint8_t *codes, *scales;         // the output in 8 bits
    int64_t codes_stride, scales_stride;
};

// Rows of finite numbers whose squares add up beyond fp32 are taken again times 2^-80 (below 2^48 then, squares of 2^20 columns add up to less than 2^117), and rows whose mean square
// is so small that squares have lost bits, and that eps does not outweigh, times 2^90.
constexpr float kRmsDown = 0x1p-80f, kRmsUp = 0x1p90f, kRmsLeast = 0x1p-100f;
template <typename T>
__device__ __forceinline__ bool rms_far(float mean_square, float eps) {
    return kFarRows<T> && (!(mean_square < INFINITY) || (mean_square < kRmsLeast && eps < kRmsLeast));
}

template <typename T>
__device__ __forceinline__ float rms_sum(const T *x, const T *res, int64_t c) { return (float)(res ? (T)((float)x[c] + (float)res[c]) : x[c]); }

// y of one column of a row that is taken again; a block's 32 columns are 32 adjacent lanes' (all of them come here)
template <typename T, bool OUT8>
__device__ __forceinline__ void rms_put(const RmsArgs &a, int64_t row, int c, bool here, float y) {
    if (!OUT8) {
        if (here) ((T *)a.y)[row * a.d + c] = (T)y;
        return;
    }
    const uint32_t byte = scale_byte(lanes_max<kScaleBlock>(here ? finite_amount(y) : 0.f));
    if (!here) return;
    a.codes[row * a.codes_stride + c] = (uint8_t)to_fp8(y * scale_inverse(byte), 0.f, 0.f, 0.f);
    if (c % kScaleBlock == 0) a.scales[row * a.scales_stride + c / kScaleBlock] = (uint8_t)byte;
}

// A row out of fp32's range (`here`; other rows' lanes go along), read again by a wavefront or the workgroup: rows that nothing but a broken training meets, so what counts is that the
// ordinary ones hold no registers for them.
template <typename T, bool OUT8, int THREADS>
__device__ __forceinline__ void rms_far_row(const RmsArgs &a, int64_t row, float2 (*lds)[16], int &turn) {
    const int l = threadIdx.x % THREADS;
    const T *p = (const T *)a.x + row * a.x_stride, *q = a.res ? (const T *)a.res + row * a.res_stride : nullptr;
    float scale = kRmsDown, mean;
    for (;;) {
        float2 s = make_float2(0.f, 0.f);
#pragma unroll 1
        for (int c = l; c < a.d; c += THREADS) {
            const float v = rms_sum<T>(p, q, c) * scale;
            s.x += v * v;
        }
        mean = row_sums<THREADS>(s, lds, turn).x * a.inv_d;
        // squares that pass fp32 have a mean of at least 2^(128 - 20 - 160) here
        if (scale == kRmsUp || !(mean < 0x1p-60f)) break;
        scale = kRmsUp;
    }
    const float r = inverse_root(mean + a.eps * scale * scale);
#pragma unroll 1
    for (int c = l; c - l < a.d; c += THREADS) {
        const bool here = c < a.d;
        const float v = here ? rms_sum<T>(p, q, c) * scale * r * (a.weight ? param(a.weight, a.param32, T(), c) : 1.f) : 0.f;
        rms_put<T, OUT8>(a, row, c, here, v);
    }
    if (l == 0 && a.rstd) a.rstd[row] = r * scale;
}

// Bound by reading x and the residual and writing their sum and y.  Every lane requests R rows one after the other before it needs the first.  232965 x 128 bf16 with residual 38 us (6.2 TB/s),
// without 19.8 (6.0), 56944 x 251 fp32 20.0 (5.7).  In 8 bits 232965 x 256 bf16 with residual 75 us (5.6), 56944 x 251 fp32 16.5 (4.4: instructions issue five sixths of the time).
template <typename T, int LPR, int K, int R, bool TAIL, bool OUT8>
__global__ __launch_bounds__(kNormBlock<LPR>) void rms_kernel(RmsArgs a) {
    __shared__ float2 lds[2][16];
    typedef typename VecOf<T>::type Raw;
    constexpr int V = kVec<T>, kTaker = LPR <= kWave ? kWave : LPR;
    const int l = threadIdx.x % LPR;
    const int64_t first = ((int64_t)blockIdx.x * (kNormBlock<LPR> / kTaker) + threadIdx.x / kTaker) * (kSide<LPR> * R), row0 = first + threadIdx.x % kTaker / LPR;
    const T *x = (const T *)a.x, *res = (const T *)a.res;
    Raw raw[R][K];
    float r[R];
    uint32_t far = 0;                                      // bits of rows that are taken again
    int turn = 0;
#pragma unroll
    for (int t = 0; t < R; ++t) {
        const int64_t row = min(row0 + t * kSide<LPR>, a.n - 1);                   // (rows beyond the last one: that one again, not stored)
#pragma unroll
        for (int k = 0; k < K; ++k) raw[t][k] = load_columns<T, TAIL>(x, row * a.x_stride, (l + LPR * k) * V, a.d, a.x_extent);
    }
    if (res) {
        Raw more[R][K];
#pragma unroll
        for (int t = 0; t < R; ++t) {
            const int64_t row = min(row0 + t * kSide<LPR>, a.n - 1);
#pragma unroll
            for (int k = 0; k < K; ++k) more[t][k] = load_columns<T, TAIL>(res, row * a.res_stride, (l + LPR * k) * V, a.d, a.res_extent);
        }
#pragma unroll
        for (int t = 0; t < R; ++t)
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int64_t row = row0 + t * kSide<LPR>;
                const int col = (l + LPR * k) * V;
                float h[V];
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    h[e] = (float)raw[t][k][e] + (float)more[t][k][e];
                    raw[t][k][e] = (T)h[e];
                }
                if (row < a.n && col < a.d) store_vec((T *)a.h + row * a.d + col, TAIL ? a.d - col : V, h);
            }
    }
#pragma unroll
    for (int t = 0; t < R; ++t) {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int col = (l + LPR * k) * V;
            float part = 0.f;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float v = (float)raw[t][k][e];
                part += !TAIL || col + e < a.d ? v * v : 0.f;
            }
            s += col < a.d ? part : 0.f;
        }
        const float mean = row_sums<LPR>(make_float2(s, 0.f), lds, turn).x * a.inv_d;
        r[t] = inverse_root(mean + a.eps);
        if (rms_far<T>(mean, a.eps) && row0 + t * kSide<LPR> < a.n) far |= 1u << t;
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int col = (l + LPR * k) * V;
        float w[V];
        load_params<T, TAIL>(a.weight, a.param32, col, a.d, 1.f, w);
#pragma unroll
        for (int t = 0; t < R; ++t) {
            const int64_t row = row0 + t * kSide<LPR>;
            const bool here = row < a.n && col < a.d && !(far >> t & 1);
            float y[V];
#pragma unroll
            for (int e = 0; e < V; ++e) y[e] = (float)raw[t][k][e] * r[t] * w[e];
            if (!OUT8) {
                if (here) store_vec((T *)a.y + row * a.d + col, TAIL ? a.d - col : V, y);
                continue;
            }
            constexpr int kLanes = LPR < kScaleBlock / V ? LPR : kScaleBlock / V;   // of a block
            uint32_t most = 0;                             // as whole numbers, those that are none are above all others
#pragma unroll
            for (int e = 0; e < V; ++e) most = max(most, (TAIL ? col + e : col) < a.d ? __float_as_uint(y[e]) & 0x7fffffffu : 0u);
            if (__any(most >= 0x7f800000u)) {
                most = 0;
#pragma unroll
                for (int e = 0; e < V; ++e) most = max(most, (TAIL ? col + e : col) < a.d ? __float_as_uint(finite_amount(y[e])) : 0u);
            }
            const uint32_t byte = scale_byte(lanes_max<kLanes>(__uint_as_float(most)));
            const float by = scale_inverse(byte);
            if (!here) continue;
            uint32_t code[V / 4];
#pragma unroll
            for (int e = 0; e < V; e += 4) code[e / 4] = to_fp8(y[e] * by, y[e + 1] * by, y[e + 2] * by, y[e + 3] * by);
            uint8_t *to = a.codes + row * a.codes_stride + col;
            if (!TAIL || col + V <= a.d) {
                typedef uint32_t code_t __attribute__((ext_vector_type(V / 4), aligned(1)));
                code_t packed;
#pragma unroll
                for (int e = 0; e < V / 4; ++e) packed[e] = code[e];
                *reinterpret_cast<code_t *>(to) = packed;
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e)
                    if (col + e < a.d) to[e] = (uint8_t)(code[e / 4] >> 8 * (e % 4));
            }
            if (l % kLanes == 0) a.scales[row * a.scales_stride + col / kScaleBlock] = (uint8_t)byte;
        }
    }
    if (a.rstd && l == 0) {
#pragma unroll
        for (int t = 0; t < R; ++t) {
            const int64_t row = row0 + t * kSide<LPR>;
            if (row < a.n && !(far >> t & 1)) a.rstd[row] = r[t];
        }
    }
    if (kFarRows<T> && __any(far != 0)) {                  // (a row of more than a wavefront: the same in all of them)
#pragma unroll 1
        for (int t = 0; t < R; ++t)
#pragma unroll 1
            for (int side = 0; side < kSide<LPR>; ++side)
                if (__shfl((int)(far >> t & 1), side * (LPR < kWave ? LPR : 0))) rms_far_row<T, OUT8, kTaker>(a, first + t * kSide<LPR> + side, lds, turn);
    }
}

// Rows that registers do not hold: a workgroup of 1024 reads its row again.
template <typename T, bool OUT8>
__global__ __launch_bounds__(kWide) void rms_wide_kernel(RmsArgs a) {
    __shared__ float2 lds[2][16];
    const int64_t row = blockIdx.x;
    const T *p = (const T *)a.x + row * a.x_stride, *q = a.res ? (const T *)a.res + row * a.res_stride : nullptr;
    int turn = 0;
    float2 s = make_float2(0.f, 0.f);
    for (int c = threadIdx.x; c < a.d; c += kWide) {
        const float v = rms_sum<T>(p, q, c);
        if (q) ((T *)a.h)[row * a.d + c] = (T)v;
        s.x += v * v;
    }
    const float mean = row_sums<kWide>(s, lds, turn).x * a.inv_d;
    if (rms_far<T>(mean, a.eps)) {
        rms_far_row<T, OUT8, kWide>(a, row, lds, turn);
        return;
    }
    const float r = inverse_root(mean + a.eps);
    const T *sum = q ? (const T *)a.h + row * a.d : p;     // (every thread reads the columns that it wrote)
    for (int c = threadIdx.x; c - (int)threadIdx.x < a.d; c += kWide) {
        const bool here = c < a.d;
        const float v = here ? (float)sum[c] * r * (a.weight ? param(a.weight, a.param32, T(), c) : 1.f) : 0.f;
        rms_put<T, OUT8>(a, row, c, here, v);
    }
    if (threadIdx.x == 0 && a.rstd) a.rstd[row] = r;
}

typedef void (*rms_kernel_t)(RmsArgs);
template <typename T>
static int rms_launch(rms_kernel_t kernel, const RmsArgs &a, int64_t rows, int threads, hipStream_t s) {
    return launch_parts((a.n + rows - 1) / rows, threads, [&](int64_t first, int64_t count) {
        const int64_t at = first * rows;
        RmsArgs part = a;
        part.n = std::min(count * rows, a.n - at);
        part.x = (const T *)a.x + at * a.x_stride;
        part.x_extent = (part.n - 1) * a.x_stride + a.d;
        part.res = a.res ? (const T *)a.res + at * a.res_stride : nullptr;
        part.res_extent = (part.n - 1) * a.res_stride + a.d;
        part.h = a.h ? (T *)a.h + at * a.d : nullptr;
        part.y = a.y ? (T *)a.y + at * a.d : nullptr;
        part.rstd = a.rstd ? a.rstd + at : nullptr;
        part.codes = a.codes ? a.codes + at * a.codes_stride : nullptr;
        part.scales = a.scales ? a.scales + at * a.scales_stride : nullptr;
        hipLaunchKernelGGL(kernel, dim3((unsigned)count), dim3((unsigned)threads), 0, s, part);
    });
}
// Rows one after the other that a lane requests at once: 16 columns' worth.
constexpr int rms_rows(int lpr, int k, int vec) { return lpr > kWave || k * vec >= 16 ? 1 : 16 / (k * vec); }
template <typename T, bool TAIL, bool OUT8>
struct RmsForward {
    template <int LPR, int K>
    struct Of { static constexpr auto kernel = rms_kernel<T, LPR, K, rms_rows(LPR, K, kVec<T>), TAIL, OUT8>; };
};

struct RmsGradArgs {
    const void *h, *gy, *gh;         // gh: the gradient that arrives at h by itself, or NULL
    int64_t h_stride, gy_stride, gh_stride, n;
    int64_t h_extent, gy_extent, gh_extent;
    int32_t d, param32;
    const void *weight;              // or NULL
    const float *rstd;
    float inv_d;
    void *gx;                        // contiguous
    float *partial;                  // g_w of every workgroup [groups, d]; NULL: not wanted, or one workgroup does it all
    void *g_w;                       // for one workgroup
};

// Bound by reading h, g_y and g_h and writing g_x.  Workgroups take rows in turn, keep the sums of their columns for g_w in registers, and leave them in `partial`, added up in a fixed
// order by rms_reduce_kernel.  The next rows are requested before the present ones are worked on.  65536 x 512 fp32 with g_h 100 us with the last sums (5.3 TB/s), 56944 x 251 bf16 20.7 (4.1).
template <typename T, int LPR, int K, int R, bool TAIL>
__global__ __launch_bounds__(kGradBlock<LPR>) void rms_grad_kernel(RmsGradArgs a) {
    extern __shared__ float sums[];                        // [wavefronts][LPR * K * V], rows of up to 64 lanes
    __shared__ float2 lds[2][16];
    typedef typename VecOf<T>::type Raw;
    constexpr int V = kVec<T>, kTaker = LPR <= kWave ? kWave : LPR, kTakers = kGradBlock<LPR> / kTaker;   // what takes a set of rows: a wavefront, or the workgroup
    const int l = threadIdx.x % LPR, side = threadIdx.x % kTaker / LPR;
    const T *h = (const T *)a.h, *gy = (const T *)a.gy, *gh = (const T *)a.gh;
    int turn = 0;
    float w[K][V], gw[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        load_params<T, TAIL>(a.weight, a.param32, (l + LPR * k) * V, a.d, 1.f, w[k]);
#pragma unroll
        for (int e = 0; e < V; ++e) gw[k][e] = 0.f;
    }
    const int64_t sets = (a.n + kSide<LPR> * R - 1) / (kSide<LPR> * R), step = (int64_t)gridDim.x * kTakers;
    struct Rows {
        Raw h[R][K], g[R][K], more[R][K];
        float r[R];
    };
    auto request = [&](int64_t set, Rows &q) {
#pragma unroll
        for (int t = 0; t < R; ++t) {
            const int64_t row = min((set * R + t) * kSide<LPR> + side, a.n - 1);
            q.r[t] = a.rstd[row];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                q.h[t][k] = load_columns<T, TAIL>(h, row * a.h_stride, (l + LPR * k) * V, a.d, a.h_extent);
                q.g[t][k] = load_columns<T, TAIL>(gy, row * a.gy_stride, (l + LPR * k) * V, a.d, a.gy_extent);
                if (gh) q.more[t][k] = load_columns<T, TAIL>(gh, row * a.gh_stride, (l + LPR * k) * V, a.d, a.gh_extent);
            }
        }
    };
    auto work = [&](int64_t set, const Rows &q) {
#pragma unroll
        for (int t = 0; t < R; ++t) {
            const int64_t row = (set * R + t) * kSide<LPR> + side;
            const bool here = row < a.n;
            float s = 0.f, xh[K][V], u[K][V];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int col = (l + LPR * k) * V;
                float part = 0.f;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const bool in = here && (!TAIL || col + e < a.d);
                    const float g = in ? (float)q.g[t][k][e] : 0.f;
                    xh[k][e] = in ? (float)q.h[t][k][e] * q.r[t] : 0.f;
                    u[k][e] = g * w[k][e];
                    gw[k][e] += g * xh[k][e];              // (columns beyond the row's end: not read)
                    part += u[k][e] * xh[k][e];
                }
                s += col < a.d ? part : 0.f;
            }
            s = row_sums<LPR>(make_float2(s, 0.f), lds, turn).x * a.inv_d;
            if (!here) continue;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int col = (l + LPR * k) * V;
                if (col >= a.d) continue;
#pragma unroll
                for (int e = 0; e < V; ++e) u[k][e] = q.r[t] * (u[k][e] - xh[k][e] * s);
                if (gh) {
#pragma unroll
                    for (int e = 0; e < V; ++e) u[k][e] += (float)q.more[t][k][e];
                }
                store_vec((T *)a.gx + row * a.d + col, TAIL ? a.d - col : V, u[k]);
            }
        }
    };
    int64_t set = (int64_t)blockIdx.x * kTakers + threadIdx.x / kTaker;
    if (set < sets) {
        Rows q = {};
        request(set, q);
        for (; set < sets; set += step) {
            Rows next = q;
            if (set + step < sets) request(set + step, next);
            work(set, q);
            q = next;
        }
    }
    if (!a.partial && !a.g_w) return;
    auto leave = [&](int c, float sum) {
        if (a.partial) a.partial[(int64_t)blockIdx.x * a.d + c] = sum;
        else if (a.param32) ((float *)a.g_w)[c] = sum;
        else ((T *)a.g_w)[c] = (T)sum;
    };
    if (LPR > kWave) {                                     // every column has one lane
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int e = 0; e < V; ++e)
                if ((l + LPR * k) * V + e < a.d) leave((l + LPR * k) * V + e, gw[k][e]);
        return;
    }
    // lanes that hold the same columns, then the wavefronts in their order
    constexpr int kWidth = LPR * K * V;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e)
#pragma unroll
            for (int off = LPR; off < kWave; off <<= 1) gw[k][e] += __shfl_xor(gw[k][e], off);
    if (threadIdx.x % kWave < LPR) {
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int e = 0; e < V; ++e) sums[threadIdx.x / kWave * kWidth + (l + LPR * k) * V + e] = gw[k][e];
    }
    __syncthreads();
    for (int c = threadIdx.x; c < a.d; c += kGradBlock<LPR>) {
        float sum = 0.f;
#pragma unroll
        for (int wave = 0; wave < kTakers; ++wave) sum += sums[wave * kWidth + c];
        leave(c, sum);
    }
}

// g_w: 16 columns per workgroup, 64 threads for each, which take every 64th row of `partial`, then those in a fixed order
template <typename P>
__global__ __launch_bounds__(1024) void rms_reduce_kernel(const float *__restrict__ partial, int32_t groups, int32_t d, P *__restrict__ g_w) {
    __shared__ float part[64][17];
    const int o = threadIdx.x & 15, p = threadIdx.x >> 4, i = blockIdx.x * 16 + o;
    float sum = 0.f;
    if (i < d) {
#pragma unroll 8
        for (int g = p; g < groups; g += 64) sum += partial[(int64_t)g * d + i];
    }
    part[p][o] = sum;
    __syncthreads();
    for (int half = 32; half > 0; half >>= 1) {
        if (p < half) part[p][o] += part[p + half][o];
        __syncthreads();
    }
    if (p == 0 && i < d) g_w[i] = (P)part[0][o];
}

template <typename T>
__global__ __launch_bounds__(kWide) void rms_grad_wide_kernel(RmsGradArgs a) {
    __shared__ float2 lds[2][16];
    const int64_t row = blockIdx.x;
    const T *p = (const T *)a.h + row * a.h_stride, *g = (const T *)a.gy + row * a.gy_stride, *more = a.gh ? (const T *)a.gh + row * a.gh_stride : nullptr;
    const float r = a.rstd[row];
    int turn = 0;
    float2 s = make_float2(0.f, 0.f);
    for (int c = threadIdx.x; c < a.d; c += kWide) s.x += (float)g[c] * (a.weight ? param(a.weight, a.param32, T(), c) : 1.f) * ((float)p[c] * r);
    const float mean = row_sums<kWide>(s, lds, turn).x * a.inv_d;
    for (int c = threadIdx.x; c < a.d; c += kWide) {
        const float u = (float)g[c] * (a.weight ? param(a.weight, a.param32, T(), c) : 1.f);
        ((T *)a.gx)[row * a.d + c] = (T)(r * (u - (float)p[c] * r * mean) + (more ? (float)more[c] : 0.f));
    }
}

// partial[slice] = the sums of a slice of the rows, 64 columns per workgroup
template <typename T>
__global__ __launch_bounds__(kBlock) void rms_wide_sums_kernel(RmsGradArgs a) {
    __shared__ float lds[kBlock / kWave][kWave];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, c = blockIdx.x * kWave + lane;
    float gw = 0.f;
    if (c < a.d) {
        for (int64_t row = (int64_t)blockIdx.y * (kBlock / kWave) + wave; row < a.n; row += (int64_t)gridDim.y * (kBlock / kWave))
            gw += (float)((const T *)a.gy)[row * a.gy_stride + c] * ((float)((const T *)a.h)[row * a.h_stride + c] * a.rstd[row]);
    }
    lds[wave][lane] = gw;
    __syncthreads();
    if (wave > 0 || c >= a.d) return;
    for (int v = 1; v < kBlock / kWave; ++v) gw += lds[v][lane];
    a.partial[(int64_t)blockIdx.y * a.d + c] = gw;
}

typedef void (*rms_grad_kernel_t)(RmsGradArgs);
constexpr int rms_grad_rows(int lpr, int k) { return lpr <= kWave && k == 1 ? 2 : 1; }
template <typename T, bool TAIL>
struct RmsBackward {
    template <int LPR, int K>
    struct Of { static constexpr auto kernel = rms_grad_kernel<T, LPR, K, rms_grad_rows(LPR, K), TAIL>; };
};

// Workgroups of a backward pass: one for each of the 256 compute units, so that few partial sums are written and read again; two where rows are shorter than a wavefront.
constexpr int64_t kRmsSlices = 128;
static int64_t rms_grad_groups(int64_t n, NormShape s) {
    if (s.k == 0) return kRmsSlices;
    const int64_t rows = s.lpr <= kWave ? norm_side(s, true) * rms_grad_rows(s.lpr, s.k) * 4 : 8;
    return std::max<int64_t>(1, std::min<int64_t>((n + rows - 1) / rows, s.lpr < kWave ? 512 : 256));
}

static const char *rms_refusal(int64_t n, int64_t d, hag_dtype_t dtype, hag_dtype_t param_dtype) {
    if (n < 0 || d <= 0 || n > 0x7fffffffLL || d > (1 << 20)) return "n must be in 0 .. 2^31 - 1, d in 1 .. 2^20";
    if (!elem_type(dtype)) return "elements are HAG_F32, HAG_BF16 or HAG_F16";
    if (param_dtype != dtype && param_dtype != HAG_F32) return "weight has the elements' type or HAG_F32";
    return nullptr;
}

// What the two forward calls have in common; nothing to do where args.n is 0 afterwards.
static int rms_args(int64_t n, int64_t d, hag_dtype_t dtype, const void *x, int64_t x_stride, const void *residual, int64_t residual_stride, hag_dtype_t param_dtype, const void *weight,
                    float eps, void *h, RmsArgs &a) {
    if (const char *why = rms_refusal(n, d, dtype, param_dtype)) { set_error(why); return HAG_EINVAL; }
    if (x_stride < 0 || residual_stride < 0) { set_error("negative row stride"); return HAG_EINVAL; }
    if (!(eps >= 0.f) || !(eps < INFINITY)) { set_error("eps must be a number and not negative"); return HAG_EINVAL; }
    a = {};
    if (n == 0) return HAG_OK;
    if (!x || (residual && !h)) { set_error("NULL pointer"); return HAG_EINVAL; }
    a.x = x;
    a.res = residual;
    a.x_stride = x_stride;
    a.res_stride = residual_stride;
    a.n = n;
    a.x_extent = (n - 1) * x_stride + d;
    a.res_extent = (n - 1) * residual_stride + d;
    a.d = (int32_t)d;
    a.param32 = param_dtype == HAG_F32;
    a.weight = weight;
    a.eps = eps;
    a.inv_d = 1.f / (float)d;
    a.h = residual ? h : nullptr;
    return HAG_OK;
}

// Rows whose output has 8 bits are bound by instructions rather than bytes: half a wavefront, of two vectors a lane, halves what is done once a lane and row (56944 x 251 fp32 18.5 -> 16.3 us,
// x 256 14.3 -> 13.8; fewer lanes for shorter rows gain nothing: 232965 x 100 22.7 -> 23.9).
static NormShape rms_shape(int64_t d, int vec, bool out8) {
    const NormShape s = norm_shape(d, vec);
    return out8 && s.lpr == kWave && s.k == 1 ? NormShape{kWave / 2, 2} : s;
}

template <bool OUT8>
static int rms_forward(const RmsArgs &a, hag_dtype_t dtype, hipStream_t stream) {
    return elem_switch(dtype, [&](auto e) {
        using T = decltype(e);
        const NormShape s = rms_shape(a.d, kVec<T>, OUT8);
        if (s.k == 0) return rms_launch<T>(rms_wide_kernel<T, OUT8>, a, 1, kWide, stream);
        rms_kernel_t kernel;
        if (OUT8 && s.lpr == kWave / 2 && s.k == 2) kernel = a.d % kVec<T> ? RmsForward<T, true, true>::template Of<32, 2>::kernel : RmsForward<T, false, true>::template Of<32, 2>::kernel;
        else kernel = a.d % kVec<T> ? norm_pick<rms_kernel_t, T, RmsForward<T, true, OUT8>::template Of>(s) : norm_pick<rms_kernel_t, T, RmsForward<T, false, OUT8>::template Of>(s);
        return rms_launch<T>(kernel, a, norm_side(s, false) * rms_rows(s.lpr, s.k, kVec<T>), norm_block(s, false), stream);
    });
}

}  // namespace hag

using namespace hag;

extern "C" {

int hag_rms_norm(int64_t n, int64_t d, hag_dtype_t dtype, const void *x, int64_t x_stride, const void *residual, int64_t residual_stride, hag_dtype_t param_dtype, const void *weight,
                 float eps, void *h, void *y, float *rstd, void *stream) {
    RmsArgs a;
    if (const int rc = rms_args(n, d, dtype, x, x_stride, residual, residual_stride, param_dtype, weight, eps, h, a)) return rc;
    if (n == 0) return HAG_OK;
    if (!y) { set_error("NULL pointer"); return HAG_EINVAL; }
    a.y = y;
    a.rstd = rstd;
    return rms_forward<false>(a, dtype, (hipStream_t)stream);
}

int hag_rms_norm_fp8(int64_t n, int64_t d, hag_dtype_t dtype, const void *x, int64_t x_stride, const void *residual, int64_t residual_stride, hag_dtype_t param_dtype, const void *weight,
                     float eps, void *h, uint8_t *codes, int64_t codes_stride, uint8_t *scales, int64_t scales_stride, void *stream) {
    RmsArgs a;
    if (const int rc = rms_args(n, d, dtype, x, x_stride, residual, residual_stride, param_dtype, weight, eps, h, a)) return rc;
    if (codes_stride < d || scales_stride < (d + kScaleBlock - 1) / kScaleBlock) { set_error("rows of the output overlap"); return HAG_EINVAL; }
    if (n == 0) return HAG_OK;
    if (!codes || !scales) { set_error("NULL pointer"); return HAG_EINVAL; }
    a.codes = codes;
    a.codes_stride = codes_stride;
    a.scales = scales;
    a.scales_stride = scales_stride;
    return rms_forward<true>(a, dtype, (hipStream_t)stream);
}

size_t hag_rms_norm_grad_workspace_bytes(int64_t n, int64_t d) {
    if (rms_refusal(n, d, HAG_F32, HAG_F32)) return 0;
    // the types of 16 bits take fewer lanes to a row and no more workgroups
    return (size_t)std::max(rms_grad_groups(n, norm_shape(d, 4)), rms_grad_groups(n, norm_shape(d, 8))) * (size_t)d * sizeof(float);
}

int hag_rms_norm_grad(int64_t n, int64_t d, hag_dtype_t dtype, const void *g_y, int64_t g_y_stride, const void *g_h, int64_t g_h_stride, const void *h, int64_t h_stride,
                      hag_dtype_t param_dtype, const void *weight, const float *rstd, void *g_x, void *g_weight, void *workspace, void *stream) {
    if (const char *why = rms_refusal(n, d, dtype, param_dtype)) { set_error(why); return HAG_EINVAL; }
    if (h_stride < 0 || g_y_stride < 0 || g_h_stride < 0) { set_error("negative row stride"); return HAG_EINVAL; }
    if ((n > 0 && (!g_y || !h || !rstd || !g_x)) || (g_weight && !workspace)) { set_error("NULL pointer"); return HAG_EINVAL; }
    if ((uintptr_t)workspace & 15) { set_error("workspace must be 16-byte aligned"); return HAG_EINVAL; }
    if (n == 0 && !g_weight) return HAG_OK;
    hipStream_t s = (hipStream_t)stream;
    RmsGradArgs a = {};
    a.h = h;
    a.gy = g_y;
    a.gh = g_h;
    a.h_stride = h_stride;
    a.gy_stride = g_y_stride;
    a.gh_stride = g_h_stride;
    a.n = n;
    a.h_extent = n > 0 ? (n - 1) * h_stride + d : 0;
    a.gy_extent = n > 0 ? (n - 1) * g_y_stride + d : 0;
    a.gh_extent = n > 0 ? (n - 1) * g_h_stride + d : 0;
    a.d = (int32_t)d;
    a.param32 = param_dtype == HAG_F32;
    a.weight = weight;
    a.rstd = rstd;
    a.inv_d = 1.f / (float)d;
    a.gx = g_x;
    return elem_switch(dtype, [&](auto e) {
        using T = decltype(e);
        const NormShape shape = norm_shape(d, kVec<T>);
        const int64_t groups = rms_grad_groups(n, shape);
        if (groups > 1) a.partial = g_weight ? (float *)workspace : nullptr;
        else a.g_w = g_weight;
        if (shape.k == 0) {
            const int rc = launch_parts(n, kWide, [&](int64_t first, int64_t count) {
                RmsGradArgs part = a;
                part.n = count;
                part.h = (const T *)a.h + first * a.h_stride;
                part.gy = (const T *)a.gy + first * a.gy_stride;
                part.gh = a.gh ? (const T *)a.gh + first * a.gh_stride : nullptr;
                part.rstd = a.rstd + first;
                part.gx = (T *)a.gx + first * a.d;
                hipLaunchKernelGGL(rms_grad_wide_kernel<T>, dim3((unsigned)count), dim3(kWide), 0, s, part);
            });
            if (rc) return rc;
            if (g_weight) hipLaunchKernelGGL(rms_wide_sums_kernel<T>, dim3((unsigned)((d + kWave - 1) / kWave), (unsigned)groups), dim3(kBlock), 0, s, a);
        } else {
            const size_t lds = shape.lpr <= kWave ? (size_t)(norm_block(shape, true) / kWave) * shape.lpr * shape.k * kVec<T> * sizeof(float) : 0;
            const rms_grad_kernel_t kernel = d % kVec<T> ? norm_pick<rms_grad_kernel_t, T, RmsBackward<T, true>::template Of>(shape)
                                                         : norm_pick<rms_grad_kernel_t, T, RmsBackward<T, false>::template Of>(shape);
            hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3((unsigned)norm_block(shape, true)), lds, s, a);
        }
        HIP_TRY(hipGetLastError());
        if (!a.partial) return (int)HAG_OK;
        const dim3 grid((unsigned)((d + 15) / 16)), block(1024);
        if (a.param32) hipLaunchKernelGGL(rms_reduce_kernel<float>, grid, block, 0, s, a.partial, (int32_t)groups, (int32_t)d, (float *)g_weight);
        else hipLaunchKernelGGL(rms_reduce_kernel<T>, grid, block, 0, s, a.partial, (int32_t)groups, (int32_t)d, (T *)g_weight);
        HIP_TRY(hipGetLastError());
        return (int)HAG_OK;
    });
}

}  // extern "C"
