// y = x w^T for rows x [n, d] and w [k, d] in 8 bits with a power of two for every 32 columns: y_ij = sum over blocks b of 2^(sx_ib + sw_jb - 254) sum over c in b of x_ic w_jc.
// The rows of w are the matrix instructions' rows, so a lane gets four consecutive columns of y.
// A result of 16 bits takes the elements as they are, 128 columns at a time (v_mfma_scale_f32_16x16x128_f8f6f4): lane l brings, of row l % 16 of either operand, columns 16 q .. 16 q + 15 and
// 64 + 16 q .. 79 + 16 q, q = l / 16, and the scale of columns 32 q .. 32 q + 31.  Sums are kept in fp32, but before they are added the 8 products that a lane brings next to each other
// are cut off at 2^-13 of the power of two of the largest of them, an element below 2^-6 of its scale counting as 2^-6 (measured: randn operands are off by 1.5e-5 of the result's norm, 5e-5
// where elements differ by powers of e^2; the instruction for 32 columns without scales is the same): little beside the rounding to 8 or 11 bits, and for small elements 2^-9 of what their own
// rounding, to 2^-10 of the scale, left off.
// An fp32 result takes them as bf16 numbers, which hold an element times its scale exactly, 32 columns at a time (v_mfma_f32_16x16x32_bf16): products are exact, sums as good as in fp32 one
// by one (5e-8 and 3e-7 of the norm at 2048 columns), at half of the rate.  Which columns meet in an instruction is free, so lanes bring the same 16 columns either way.
#include "hag_fp8.hpp"

namespace hag {

struct ProductArgs {
    const uint8_t *x, *w, *x_scales, *w_scales;
    int64_t x_stride, w_stride, x_scales_stride, w_scales_stride;   // bytes
    int64_t n, k;
    int32_t d;
    void *y;                         // contiguous
};

typedef int frag_t __attribute__((ext_vector_type(8)));
typedef __bf16 wide_t __attribute__((ext_vector_type(8)));
typedef __bf16 wide2_t __attribute__((ext_vector_type(2)));
typedef float sums_t __attribute__((ext_vector_type(4)));
typedef uint32_t bytes16_t __attribute__((ext_vector_type(4), aligned(1)));

// The scale of a block, 1 beyond the last
__device__ __forceinline__ uint32_t load_scale(const uint8_t *row, int block, int d) { return block * kScaleBlock < d ? row[block] : 127u; }

// 128 columns of a row, as far as a lane brings them: two pieces of 16, in the types of the instruction
template <bool WIDE>
struct Part;
template <>
struct Part<false> {
    frag_t f;
    int scale;
    Part() = default;
    // scales: of the lane's blocks in its bytes, the one of columns 32 q first
    __device__ __forceinline__ Part(const bytes16_t &a, const bytes16_t &b, uint32_t scales) : scale((int)scales) {
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[i] = (int)a[i]; f[i + 4] = (int)b[i]; }
    }
};
template <>
struct Part<true> {
    wide_t f[4];
    Part() = default;
    // scales: of the two pieces in the two lower bytes
    __device__ __forceinline__ Part(const bytes16_t &a, const bytes16_t &b, uint32_t scales) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const float scale = __uint_as_float((half ? scales >> 8 & 0xffu : scales & 0xffu) << 23);   // (only its exponent counts)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t v = half ? b[i] : a[i];
                const wide2_t low = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, scale, false), high = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, scale, true);
                wide_t &to = f[half * 2 + i / 2];
                to[i % 2 * 4] = low.x;
                to[i % 2 * 4 + 1] = low.y;
                to[i % 2 * 4 + 2] = high.x;
                to[i % 2 * 4 + 3] = high.y;
            }
        }
    }
};
// A lane's scales out of the four of 128 columns
template <bool WIDE>
__device__ __forceinline__ uint32_t lane_scales(uint32_t four, int q) {
    if (!WIDE) return four >> 8 * q;
    const uint32_t mine = four >> 8 * (q / 2);             // blocks q / 2 and q / 2 + 2
    return (mine & 0xffu) | (mine >> 8 & 0xff00u);
}

// acc[0 .. T) += w x for the T pieces of w; one instruction's sums are not waited for by the next
template <int T>
__device__ __forceinline__ void multiply(const Part<false> (&w)[T], const Part<false> &x, sums_t (&acc)[T]) {
#pragma unroll
    for (int t = 0; t < T; ++t) acc[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w[t].f, x.f, acc[t], 0, 0, 0, w[t].scale, 0, x.scale);
}
template <int T>
__device__ __forceinline__ void multiply(const Part<true> (&w)[T], const Part<true> &x, sums_t (&acc)[T]) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int t = 0; t < T; ++t) acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[t].f[i], x.f[i], acc[t], 0, 0, 0);
}

// Which row of w is row m of piece t, so that a store of 16 bytes by the 4 lanes of a row of y writes 64 adjacent bytes: lanes have 4 adjacent columns of a piece; where 16 bytes are 8
// columns, pieces take turns of 4.
template <typename O>
__device__ __forceinline__ int piece_column(int t, int m) { return kVec<O> == 4 ? t * 16 + m : t / 2 * 32 + m / 4 * 8 + t % 2 * 4 + m % 4; }
// A lane's columns of the T pieces, q = lane / 16, to the row of y at `to`, of which `have` columns are there
template <typename O, int T>
__device__ __forceinline__ void store_columns(O *to, int q, int have, const sums_t (&acc)[T]) {
    constexpr int V = kVec<O>, P = V / 4;
#pragma unroll
    for (int t = 0; t < T; t += P) {
        const int col = t * 16 + q * V;
        float v[V];
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = acc[t + e / 4][e % 4];
        if (col < have) store_vec(to + col, have - col, v);
    }
}

// ------------------------------------------------------------------------------------------------ tiles through LDS

// 16 zeros, for columns beyond the last
__device__ const uint4 kNoColumns = {0, 0, 0, 0};

// Where piece `chunk` (16 columns) of a row of 128 lies in LDS: lanes that read the same piece of adjacent rows meet different banks.  w is read in the order of piece_column.
template <typename O, bool W>
__device__ __forceinline__ int placed(int row, int chunk) { return row * 8 + (chunk ^ (W && kVec<O> == 8 ? (row & 3) | (row >> 3 & 1) << 2 : row & 7)); }

struct ProductTiles {
    ProductArgs p;
    int32_t col_tiles, tiles;
};

// A workgroup takes TM rows of x and TN of w, its wavefronts WR times WC parts of them.  128 columns of both are on their way from memory to LDS, past the registers, while the 128 before are
// multiplied; the first two sets are requested together.  What LDS holds and the registers' sums limit the tile: 256 x 256 for results of 16 bits (64 KB for 128 columns, two of them; 128
// registers of sums).
// 131072 x 1024 x 1024 into bf16 186 us in hundreds of passes without a pause (1.48 PFLOP/s; the library's bf16 product of these sizes 253 us), 204 in 15 passes after one (303).  Of 200 in such
// short runs it takes 190 without the products, 142 without the stores, 163 without the loads: loads come 2 us after they are asked for, and only as much is on its way as LDS has room for.
// There, 128 columns as two 64s, so that two workgroups fit a compute unit, took 266 (lines of 128 bytes are asked for twice, what L2 answers per clock), one workgroup that goes from tile to
// tile and asks for the next one's first columns early 212, tiles of 128 x 128 259.
// Narrow results are bound by memory (without pauses): 232965 x 128 x 128 into bf16 17.3 us (5.2 TB/s), into fp32 28.0 (5.4), 56944 x 251 x 74 into fp32 11.5 (2.8: a load's way, a product's, a
// store's).
// fp32 results convert in registers: 131072 x 1024 x 1024 326 us without pauses (0.84 PFLOP/s), 390 after one (in one run 362, and 364 with the next piece converted between the products of the
// present one), 16384 x 2048 x 2048 134 (1.02) and 153.
template <typename O, int TM, int TN, int WR, int WC>
__global__ __launch_bounds__(kWave * WR * WC, 2) void product_tile_kernel(ProductTiles args) {
    constexpr bool WIDE = sizeof(O) == 4;
    constexpr int THREADS = kWave * WR * WC, ROWS = TM + TN, LOADS = ROWS * 8 / THREADS, X_LOADS = TM * 8 / THREADS, R = TM / WR / 16, T = TN / WC / 16, SCALES = (ROWS + THREADS - 1) / THREADS;
    static_assert(TM * 8 % THREADS == 0 && ROWS * 8 % THREADS == 0, "a load is of x or of w");
    // (arrays of their own, and code of its own for either: what is on its way to one is not waited for before the other is read)
    __shared__ bytes16_t codes0[ROWS * 8] __attribute__((aligned(16))), codes1[ROWS * 8] __attribute__((aligned(16)));
    __shared__ uint32_t scales0[ROWS], scales1[ROWS];
    const ProductArgs &a = args.p;
    // consecutive workgroups go to the 8 XCDs in turn: each XCD gets consecutive tiles, so that the tiles of one set of rows find them in its L2
    const int share = (args.tiles + 7) / 8, tile = (int)(blockIdx.x % 8) * share + (int)(blockIdx.x / 8);
    if ((int)(blockIdx.x / 8) >= share || tile >= args.tiles) return;
    const int64_t row0 = (int64_t)(tile / args.col_tiles) * TM, col0 = (int64_t)(tile % args.col_tiles) * TN;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, r = lane % 16, q = lane / 16, wr = wave / WC, wc = wave % WC;
    const uint8_t *x = a.x + row0 * a.x_stride, *w = a.w + col0 * a.w_stride;
    const int x_rows = (int)min(a.n - row0, (int64_t)TM), w_rows = (int)min(a.k - col0, (int64_t)TN), steps = (a.d + 127) / 128, blocks = (a.d + kScaleBlock - 1) / kScaleBlock;
    uint32_t at[LOADS];                                    // where a thread's pieces begin
    int chunk[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int slot = i * THREADS + (int)threadIdx.x - (i < X_LOADS ? 0 : TM * 8), row = slot / 8;
        chunk[i] = i < X_LOADS ? placed<O, false>(row, slot % 8) % 8 : placed<O, true>(row, slot % 8) % 8;
        at[i] = (uint32_t)(i < X_LOADS ? min(row, x_rows - 1) * (uint32_t)a.x_stride : min(row, w_rows - 1) * (uint32_t)a.w_stride) + chunk[i] * 16;
    }
    const uint8_t *scale_row[SCALES];
#pragma unroll
    for (int i = 0; i < SCALES; ++i) {
        const int row = min(i * THREADS + (int)threadIdx.x, ROWS - 1);
        scale_row[i] = row < TM ? a.x_scales + (row0 + min(row, x_rows - 1)) * a.x_scales_stride : a.w_scales + (col0 + min(row - TM, w_rows - 1)) * a.w_scales_stride;
    }
    uint32_t scale0[SCALES], scale1[SCALES];
    auto request = [&](int step, bytes16_t *codes, uint32_t (&scale)[SCALES]) {
        const uint8_t *from_x = x + (int64_t)step * 128, *from_w = w + (int64_t)step * 128;
        auto load = [&](const uint8_t *from, int i) {
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from, (__attribute__((address_space(3))) void *)(codes + i * THREADS + wave * kWave), 16, 0, 0);
        };
        if ((step + 1) * 128 <= a.d) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) load((i < X_LOADS ? from_x : from_w) + at[i], i);
        } else {                                           // (a piece that the row ends in is read to its end: it is aligned, so its other bytes are memory too)
#pragma unroll
            for (int i = 0; i < LOADS; ++i) load(step * 128 + chunk[i] * 16 < a.d ? (i < X_LOADS ? from_x : from_w) + at[i] : (const uint8_t *)&kNoColumns, i);
        }
#pragma unroll
        for (int i = 0; i < SCALES; ++i) {
            typedef uint32_t word_t __attribute__((aligned(1)));
            if (step * 4 + 4 <= blocks) {
                scale[i] = *reinterpret_cast<const word_t *>(scale_row[i] + step * 4);
            } else {
                scale[i] = 0x7f7f7f7fu;
#pragma unroll
                for (int b = 0; b < 3; ++b)
                    if (step * 4 + b < blocks) scale[i] = (scale[i] & ~(0xffu << 8 * b)) | (uint32_t)scale_row[i][step * 4 + b] << 8 * b;
            }
        }
    };
    auto keep_scales = [&](uint32_t *scales, const uint32_t (&scale)[SCALES]) {
#pragma unroll
        for (int i = 0; i < SCALES; ++i)
            if (SCALES * THREADS == ROWS || i * THREADS + (int)threadIdx.x < ROWS) scales[i * THREADS + threadIdx.x] = scale[i];
    };
    sums_t acc[R][T];
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
        for (int t = 0; t < T; ++t) acc[i][t] = sums_t{0.f, 0.f, 0.f, 0.f};
    // what the row's last piece has beyond its end becomes zeros, by the thread that brought it
    auto cut = [&](int step, bytes16_t *codes) {
        __builtin_amdgcn_s_waitcnt(0);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int have = a.d - step * 128 - chunk[i] * 16;
            if (have <= 0 || have >= 16) continue;
            bytes16_t &v = codes[i * THREADS + threadIdx.x];
#pragma unroll
            for (int b = 0; b < 4; ++b) v[b] &= have >= 4 * b + 4 ? ~0u : have <= 4 * b ? 0u : (1u << 8 * (have - 4 * b)) - 1u;
        }
    };
    // (rows 16 apart of x, and w's as piece_column puts them, have their pieces in the same places)
    static_assert(T == 4, "pieces of w are placed for 64 columns of a wavefront");
    const int x_row = wr * (TM / WR) + r, w_row = wc * (TN / WC) + piece_column<O>(0, r);
    const int x_a = placed<O, false>(x_row, q), x_b = placed<O, false>(x_row, q + 4), w_a = TM * 8 + placed<O, true>(w_row, q), w_b = TM * 8 + placed<O, true>(w_row, q + 4);
    auto work = [&](const bytes16_t *of, const uint32_t *four) {
        Part<WIDE> pw[T];
#pragma unroll
        for (int t = 0; t < T; ++t) pw[t] = Part<WIDE>(of[w_a + piece_column<O>(t, 0) * 8], of[w_b + piece_column<O>(t, 0) * 8], lane_scales<WIDE>(four[TM + w_row + piece_column<O>(t, 0)], q));
        // the next piece of x is requested before the present one is multiplied, and no other: more would not fit the registers
        bytes16_t a_next = of[x_a], b_next = of[x_b];
        uint32_t four_next = four[x_row];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const Part<WIDE> px(a_next, b_next, lane_scales<WIDE>(four_next, q));
            if (i + 1 < R) {
                a_next = of[x_a + (i + 1) * 128];
                b_next = of[x_b + (i + 1) * 128];
                four_next = four[x_row + (i + 1) * 16];
            }
            multiply<T>(pw, px, acc[i]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto turn = [&](int step, bytes16_t *codes, uint32_t *scales, const uint32_t (&scale)[SCALES], bytes16_t *next, uint32_t (&next_scale)[SCALES]) {
        if (step + 1 == steps && a.d % 16) cut(step, codes);
        keep_scales(scales, scale);
        // A wavefront's own pieces have to be in LDS before the barrier lets the others read them.  Said here: a barrier waits for no load by itself, and a wavefront that keeps no scales (128 x 64:
        // one of four) has none of its own to wait for.
        __builtin_amdgcn_s_waitcnt(0x0f70);                // vmcnt(0), the other counters as they are
        __syncthreads();
        if (step > 0 && step + 1 < steps) request(step + 1, next, next_scale);
        work(codes, scales);
    };
    request(0, codes0, scale0);
    if (steps > 1) request(1, codes1, scale1);             // (both are empty: two waits become one)
    for (int step = 0; step < steps; step += 2) {
        turn(step, codes0, scales0, scale0, codes1, scale1);
        if (step + 1 < steps) turn(step + 1, codes1, scales1, scale1, codes0, scale0);
    }
    const int64_t col = col0 + wc * (TN / WC);
    const int have = (int)max((int64_t)0, min(a.k - col, (int64_t)(TN / WC)));
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int row = wr * (TM / WR) + i * 16 + r;
        if (row < x_rows) store_columns<O, T>((O *)a.y + (row0 + row) * a.k + col, q, have, acc[i]);
    }
}

// ------------------------------------------------------------------------------------------------ few rows, or rows at any address

// 16 columns from `col` of a row at any address, zeros from column d on; begin, end: of the matrix in memory.  Where 16 bytes from there are not all the matrix's, its last 16 are read and
// moved (a matrix of fewer is read byte by byte).
__device__ __forceinline__ bytes16_t load16(const uint8_t *row, int col, int d, const uint8_t *begin, const uint8_t *end) {
    bytes16_t v = {};
    const int have = d - col;
    if (have <= 0) return v;
    const uint8_t *from = row + col;
    if (have >= 16 || end - begin >= 16) {
        const int over = from > end - 16 ? (int)(from - (end - 16)) * 8 : 0;          // bits that lie beyond the end, 120 at most: from is before it
        v = *reinterpret_cast<const bytes16_t *>(over > 0 ? end - 16 : from);
        if (have < 16) {
            uint64_t low = v[0] | (uint64_t)v[1] << 32, high = v[2] | (uint64_t)v[3] << 32;
            if (over > 0) {
                low = over >= 64 ? high >> (over - 64) : low >> over | high << (64 - over);
                high = over >= 64 ? 0 : high >> over;
            }
            low &= have >= 8 ? ~0ull : (1ull << 8 * have) - 1;
            high &= have <= 8 ? 0 : (1ull << 8 * (have - 8)) - 1;
            v[0] = (uint32_t)low;
            v[1] = (uint32_t)(low >> 32);
            v[2] = (uint32_t)high;
            v[3] = (uint32_t)(high >> 32);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 15; ++i)
            if (i < have) v[i / 4] |= (uint32_t)row[col + i] << 8 * (i % 4);
    }
    return v;
}
// What a lane brings of 128 columns from `col` of a row, as it comes from memory
template <bool WIDE>
struct Raw {
    bytes16_t a, b;
    uint32_t scales;
    __device__ __forceinline__ void load(const uint8_t *row, const uint8_t *of, int col, int q, int d, const uint8_t *begin, const uint8_t *end) {
        const int block = col / kScaleBlock;
        if (col + 128 <= d) {
            a = *reinterpret_cast<const bytes16_t *>(row + col + 16 * q);
            b = *reinterpret_cast<const bytes16_t *>(row + col + 64 + 16 * q);
            scales = WIDE ? (uint32_t)of[block + q / 2] | (uint32_t)of[block + 2 + q / 2] << 8 : of[block + q];
            return;
        }
        a = load16(row, col + 16 * q, d, begin, end);
        b = load16(row, col + 64 + 16 * q, d, begin, end);
        scales = WIDE ? load_scale(of, block + q / 2, d) | load_scale(of, block + 2 + q / 2, d) << 8 : load_scale(of, block + q, d);
    }
    __device__ __forceinline__ operator Part<WIDE>() const { return Part<WIDE>(a, b, scales); }
};

// A workgroup takes 16 * R rows of x and 32 of w, its wavefronts every so many 128 columns of them, straight from memory; their sums are added up in LDS in their order.  Bound by the way
// of one load after the other to the end: 1 x 512 x 512 3.3 us, 1 x 2048 x 2048 5.5 (0.8 TB/s of weights).
template <typename O, int R>
__global__ __launch_bounds__(R == 1 ? 1024 : 512) void product_split_kernel(ProductArgs a) {
    constexpr bool WIDE = sizeof(O) == 4;
    __shared__ float4 sums[(R == 1 ? 16 : 8) * R * 2 * kWave];
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave)), waves = blockDim.x / kWave, r = lane % 16, q = lane / 16;
    const int64_t row0 = (int64_t)blockIdx.x * (16 * R), col0 = (int64_t)blockIdx.y * 32;
    const uint8_t *x[R], *x_scales[R], *w[2], *w_scales[2];
    const uint8_t *x_end = a.x + (a.n - 1) * a.x_stride + a.d, *w_end = a.w + (a.k - 1) * a.w_stride + a.d;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int64_t row = min(row0 + i * 16 + r, a.n - 1);
        x[i] = a.x + row * a.x_stride;
        x_scales[i] = a.x_scales + row * a.x_scales_stride;
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int64_t row = min(col0 + piece_column<O>(t, r), a.k - 1);
        w[t] = a.w + row * a.w_stride;
        w_scales[t] = a.w_scales + row * a.w_scales_stride;
    }
    sums_t acc[R][2];
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
        for (int t = 0; t < 2; ++t) acc[i][t] = sums_t{0.f, 0.f, 0.f, 0.f};
    Raw<WIDE> rx[R], rw[2];
    auto load = [&](int col) {
#pragma unroll
        for (int t = 0; t < 2; ++t) rw[t].load(w[t], w_scales[t], col, q, a.d, a.w, w_end);
#pragma unroll
        for (int i = 0; i < R; ++i) rx[i].load(x[i], x_scales[i], col, q, a.d, a.x, x_end);
    };
    int col = wave * 128;
    if (col < a.d) load(col);
    while (col < a.d) {
        Raw<WIDE> nx[R], nw[2];
#pragma unroll
        for (int i = 0; i < R; ++i) nx[i] = rx[i];
#pragma unroll
        for (int t = 0; t < 2; ++t) nw[t] = rw[t];
        col += waves * 128;
        if (col < a.d) load(col);                          // the next ones are on their way while these are multiplied
        const Part<WIDE> pw[2] = {nw[0], nw[1]};
#pragma unroll
        for (int i = 0; i < R; ++i) multiply<2>(pw, nx[i], acc[i]);
    }
    if (waves > 1) {
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int t = 0; t < 2; ++t) sums[((wave * R + i) * 2 + t) * kWave + lane] = make_float4(acc[i][t][0], acc[i][t][1], acc[i][t][2], acc[i][t][3]);
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
        if (i % waves != wave) continue;
        if (waves > 1) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                acc[i][t] = sums_t{0.f, 0.f, 0.f, 0.f};
                for (int v = 0; v < waves; ++v) {
                    const float4 p = sums[((v * R + i) * 2 + t) * kWave + lane];
                    acc[i][t] += sums_t{p.x, p.y, p.z, p.w};
                }
            }
        }
        const int64_t row = row0 + i * 16 + r;
        if (row < a.n) store_columns<O, 2>((O *)a.y + row * a.k + col0, q, (int)min(a.k - col0, (int64_t)32), acc[i]);
    }
}

template <typename O, int R>
static int launch_split(const ProductArgs &a, hipStream_t s) {
    const int64_t groups = (a.k + 31) / 32;
    const unsigned waves = (unsigned)std::min<int64_t>(R == 1 ? 16 : 8, (a.d + 127) / 128);
    return launch_parts((a.n + 16 * R - 1) / (16 * R), kWave * waves, [&](int64_t first, int64_t count) {
        ProductArgs part = a;
        part.x += first * (16 * R) * a.x_stride;
        part.x_scales += first * (16 * R) * a.x_scales_stride;
        part.y = (O *)a.y + first * (16 * R) * a.k;
        part.n = std::min(count * (16 * R), a.n - first * (16 * R));
        hipLaunchKernelGGL((product_split_kernel<O, R>), dim3((unsigned)count, (unsigned)groups), dim3(kWave * waves), 0, s, part);
    });
}

template <typename O, int TM, int TN, int WR, int WC>
static int launch_tiles(const ProductArgs &a, hipStream_t s) {
    const int64_t col_tiles = (a.k + TN - 1) / TN, row_tiles = (a.n + TM - 1) / TM, most = std::max<int64_t>(1, ((int64_t)1 << 20) / col_tiles);
    for (int64_t first = 0; first < row_tiles; first += most) {
        const int64_t rows = std::min(most, row_tiles - first), at = first * TM;
        ProductTiles t = {a, (int32_t)col_tiles, (int32_t)(rows * col_tiles)};
        t.p.x += at * a.x_stride;
        t.p.x_scales += at * a.x_scales_stride;
        t.p.y = (O *)a.y + at * a.k;
        t.p.n = std::min(rows * TM, a.n - at);
        hipLaunchKernelGGL((product_tile_kernel<O, TM, TN, WR, WC>), dim3((unsigned)((t.tiles + 7) / 8 * 8)), dim3(kWave * WR * WC), 0, s, t);
        HIP_TRY(hipGetLastError());
    }
    return HAG_OK;
}

}  // namespace hag

using namespace hag;

extern "C" {

int hag_fp8_product(int64_t n, int64_t d, int64_t k, const uint8_t *x, int64_t x_stride, const uint8_t *x_scales, int64_t x_scales_stride, const uint8_t *w, int64_t w_stride,
                    const uint8_t *w_scales, int64_t w_scales_stride, hag_dtype_t dtype, void *y, void *stream) {
    if (n < 0 || n > 0x7fffffffLL || k < 0 || k > (1 << 20) || d <= 0 || d > (1 << 20)) { set_error("n must be in 0 .. 2^31 - 1, k in 0 .. 2^20, d in 1 .. 2^20"); return HAG_EINVAL; }
    if (!elem_type(dtype)) { set_error("the result is HAG_F32, HAG_BF16 or HAG_F16"); return HAG_EINVAL; }
    if (x_stride < 0 || w_stride < 0 || x_scales_stride < 0 || w_scales_stride < 0) { set_error("negative row stride"); return HAG_EINVAL; }
    if (n == 0 || k == 0) return HAG_OK;
    if (!x || !x_scales || !w || !w_scales || !y) { set_error("NULL pointer"); return HAG_EINVAL; }
    const ProductArgs a = {x, w, x_scales, w_scales, x_stride, w_stride, x_scales_stride, w_scales_stride, n, k, (int32_t)d, y};
    // the loads to LDS take pieces of 16 bytes at multiples of 16, and rows of a tile at 32-bit distances
    const bool aligned = !(((uintptr_t)x | (uintptr_t)w | (uintptr_t)x_stride | (uintptr_t)w_stride) & 15) && x_stride < (1 << 23) && w_stride < (1 << 23);
    return elem_switch(dtype, [&](auto e) {
        using O = decltype(e);
        hipStream_t s = (hipStream_t)stream;
        // Few workgroups: as small as they come.  64 x 2048 x 2048 into bf16: 16 rows of x each 6.8 us, 32 7.8, 64 10.8 (1 x 512 x 512 3.3, 1 x 2048 x 2048 5.5).  Up to some bytes to read
        // again they still beat tiles, which wait for memory once per 128 columns: 3000 x 2048 x 64 16 rows 10.9, 32 7.9, 64 10.8, tiles 13.6; 2000 x 256 x 256 4.2, 3.8, 3.9, 4.6;
        // 1000 x 2048 x 300 15.8, 13.1, 11.1, 14.0; but 2048 x 512 x 512 10.5, 7.9, 6.9, 6.2 and 300 x 2048 x 2048 25.9, 19.3, 20.8, 14.4.
        // Few rows of x and very many of w are tiles too: 1 x 4096 x 131072 into fp32 143 us, into bf16 125 (0.55 GB: 104).  Many rows at any address read x again for every 32 columns of y, without a
        // pause 56944 x 251 x 74 into fp32 43 us (at multiples of 16: 11.5), 232965 x 128 x 128 into bf16 109 (17.3), 131072 x 1024 x 1024 3.4 ms (186 us): whoever lays them out begins them at those.
        const int64_t groups = (k + 31) / 32, tiles = ((n + 127) / 128) * ((k + 127) / 128);
        if ((n + 15) / 16 * groups <= 256) return launch_split<O, 1>(a, s);
        if (tiles <= 64 && (n + 31) / 32 * groups * d <= 400000) return launch_split<O, 2>(a, s);
        if (!aligned || tiles <= 24) return launch_split<O, 4>(a, s);
        if (k <= 64) return launch_tiles<O, 128, 64, 4, 1>(a, s);
        // (fp32 results: 256 x 128 takes 392 us for 131072 x 1024 x 1024, 128 x 128 362; 16384 x 2048 x 2048 148 both)
        if constexpr (sizeof(O) == 2)
            if (n * k >= (int64_t)1 << 24 && k > 128) return launch_tiles<O, 256, 256, 2, 4>(a, s);
        return launch_tiles<O, 128, 128, 2, 2>(a, s);
    });
}

}  // extern "C"
