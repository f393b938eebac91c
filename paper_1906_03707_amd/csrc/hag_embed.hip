// Rows of a table looked up by id, and the gradient of the table.
//   y[i] = scale * table[id[i]],   g_table[v] = scale * (sum over the i with id[i] = v of g_y[i])
// An id equal to `padding` gives a row of zeros, one outside the table a row of NaN; neither sends a gradient.
#include "hag_elem.hpp"

namespace hag {

template <typename T, typename I>
__global__ __launch_bounds__(kBlock) void embed_kernel(const T *__restrict__ table, int64_t stride, const I *__restrict__ ids, int64_t n, int64_t rows, int32_t d,
                                                       int64_t padding, float scale, T *__restrict__ y) {
    const int lane = threadIdx.x % kWave;
    const int64_t i = (int64_t)blockIdx.x * (kBlock / kWave) + threadIdx.x / kWave;
    if (i >= n) return;
    const int64_t id = ids[i];
    const bool named = id >= 0 && id < rows && id != padding;
    for (int c = lane; c < d; c += kWave) y[i * d + c] = (T)(named ? scale * (float)table[id * stride + c] : id == padding ? 0.f : NAN);
}

// One wavefront per row of the table looks through all ids and adds up the rows of g_y that name it, in their order.
template <typename T, typename O, typename I>
__global__ __launch_bounds__(kBlock) void embed_grad_kernel(const T *__restrict__ gy, int64_t stride, const I *__restrict__ ids, int64_t n, int64_t rows, int32_t d,
                                                            int64_t padding, float scale, O *__restrict__ out) {
    const int lane = threadIdx.x % kWave;
    const int64_t v = (int64_t)blockIdx.x * (kBlock / kWave) + threadIdx.x / kWave;
    if (v >= rows) return;
    for (int c0 = 0; c0 < d; c0 += kWave) {
        const int c = c0 + lane;
        float sum = 0.f;
        for (int64_t at = 0; at < n && v != padding; at += kWave) {
            uint64_t hits = __ballot(at + lane < n && (int64_t)ids[at + lane] == v);
            for (; hits; hits &= hits - 1) {
                const int64_t i = at + __builtin_ctzll(hits);
                if (c < d) sum += (float)gy[i * stride + c];
            }
        }
        if (c < d) out[v * d + c] = (O)(scale * sum);
    }
}

}  // namespace hag

using namespace hag;

extern "C" {

// what both calls ask of their sizes
static const char *embed_refusal(int64_t n, int64_t rows, int64_t d, hag_dtype_t id_type, int64_t stride) {
    if (n < 0 || rows < 0 || d <= 0) return "n < 0, rows < 0 or d <= 0";
    if (n > 0x7fffffffLL || rows > 0x7fffffffLL - 1 || d > (1 << 20)) return "n and rows must be below 2^31, d at most 2^20";
    if (id_type != HAG_I32 && id_type != HAG_I64) return "ids are HAG_I32 or HAG_I64";
    if (stride < 0) return "negative row stride";
    return nullptr;
}

int hag_embedding(int64_t n, int64_t rows, int64_t d, hag_dtype_t dtype, const void *table, int64_t table_stride, hag_dtype_t id_type, const void *ids,
                  int64_t padding, float scale, void *y, void *stream) {
    if (const char *why = embed_refusal(n, rows, d, id_type, table_stride)) { set_error(why); return HAG_EINVAL; }
    if (!elem_type(dtype)) { set_error("elements are HAG_F32, HAG_BF16 or HAG_F16"); return HAG_EINVAL; }
    if (n == 0) return HAG_OK;
    if ((rows > 0 && !table) || !ids || !y) { set_error("NULL pointer"); return HAG_EINVAL; }
    const unsigned groups = (unsigned)((n + 3) / 4);
    return elem_switch(dtype, [&](auto e) {
        return id_switch(id_type, [&](auto k) {
            using T = decltype(e);
            using I = decltype(k);
            hipLaunchKernelGGL((embed_kernel<T, I>), dim3(groups), dim3(kBlock), 0, (hipStream_t)stream, (const T *)table, table_stride, (const I *)ids, n, rows, (int32_t)d,
                               padding, scale, (T *)y);
            HIP_TRY(hipGetLastError());
            return (int)HAG_OK;
        });
    });
}

size_t hag_embedding_grad_workspace_bytes(int64_t n, int64_t rows, int64_t d) {
    if (embed_refusal(n, rows, d, HAG_I64, 0)) return 0;
    return 16;
}

int hag_embedding_grad(int64_t n, int64_t rows, int64_t d, hag_dtype_t dtype, const void *g_y, int64_t g_y_stride, hag_dtype_t id_type, const void *ids, int64_t padding,
                       float scale, hag_dtype_t out_dtype, void *g_table, void *workspace, void *stream) {
    if (const char *why = embed_refusal(n, rows, d, id_type, g_y_stride)) { set_error(why); return HAG_EINVAL; }
    if (!elem_type(dtype) || (out_dtype != dtype && out_dtype != HAG_F32)) {
        set_error("elements are HAG_F32, HAG_BF16 or HAG_F16, those of g_table the same or HAG_F32");
        return HAG_EINVAL;
    }
    if (rows == 0) return HAG_OK;
    if ((n > 0 && (!g_y || !ids)) || !g_table || !workspace) { set_error("NULL pointer"); return HAG_EINVAL; }
    if ((uintptr_t)workspace & 15) { set_error("workspace must be 16-byte aligned"); return HAG_EINVAL; }
    return elem_switch(dtype, [&](auto e) {
        return id_switch(id_type, [&](auto k) {
            using T = decltype(e);
            using I = decltype(k);
            auto launch = [&](auto o) {
                using O = decltype(o);
                hipLaunchKernelGGL((embed_grad_kernel<T, O, I>), dim3((unsigned)((rows + 3) / 4)), dim3(kBlock), 0, (hipStream_t)stream, (const T *)g_y, g_y_stride, (const I *)ids,
                                   n, rows, (int32_t)d, padding, scale, (O *)g_table);
                HIP_TRY(hipGetLastError());
                return (int)HAG_OK;
            };
            return out_dtype == dtype ? launch(T()) : launch(float());
        });
    });
}

}  // extern "C"
