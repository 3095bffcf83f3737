// What the layer operators' part of the C ABI shares: the context, argument
// checks, workspaces.
#pragma once
#include "layer.hpp"
#include "internal.hpp"

struct dbs_layer {
    dbs::LayerWork w{};
    hipStream_t stream = nullptr;
    void *mem = nullptr;
};

inline dbs_status layer_hip_fail(hipError_t e, const char *what)
{
    (void)hipGetLastError();  // (or the next launch reports it)
    return dbs_fail(e == hipErrorOutOfMemory ? DBS_ERR_ALLOC : e == hipErrorInvalidConfiguration ? DBS_ERR_UNSUPPORTED : DBS_ERR_DEVICE, "%s: %s", what, hipGetErrorString(e));
}

#define LAYER_TRY(expr, what)                              \
    do {                                                   \
        hipError_t e_ = (expr);                            \
        if (e_ != hipSuccess) return layer_hip_fail(e_, what); \
    } while (0)

constexpr int32_t MAX_DIM = 1 << 30;

inline bool dense_type(dbs_dtype t) { return t == DBS_F16 || t == DBS_BF16; }
// One 2-D operand: rows x cols, unit column stride, `ld` elements from row to
// row.
inline dbs_status check_operand(const char *fn, const char *name, const void *p, int64_t rows, int64_t cols, int64_t ld)
{
    if (rows == 0 || cols == 0) return DBS_OK;
    if (!p) return dbs_fail(DBS_ERR_ARG, "%s: %s is NULL", fn, name);
    if ((uintptr_t)p % 2) return dbs_fail(DBS_ERR_ARG, "%s: %s is not aligned to its elements", fn, name);
    if (rows > 1 && ld < cols) return dbs_fail(DBS_ERR_ARG, "%s: %s has %lld elements from row to row, needs %lld", fn, name, (long long)ld, (long long)cols);
    if (rows > 1 && ld > (INT64_MAX / 4) / rows) return dbs_fail(DBS_ERR_UNSUPPORTED, "%s: %s spans too much memory", fn, name);
    return DBS_OK;
}
inline dbs_status check_call(const char *fn, const dbs_layer *L, dbs_dtype dt, int64_t t, int64_t n_in, int64_t n_out)
{
    if (!L) return dbs_fail(DBS_ERR_ARG, "%s: layer context is NULL", fn);
    if (!dense_type(dt)) return dbs_fail(DBS_ERR_ARG, "%s: element type must be DBS_F16 or DBS_BF16", fn);
    if (t < 0 || n_in < 0 || n_out < 0) return dbs_fail(DBS_ERR_ARG, "%s: negative size", fn);
    if (t > MAX_DIM || n_in > MAX_DIM || n_out > MAX_DIM) return dbs_fail(DBS_ERR_UNSUPPORTED, "%s: size above 2^30", fn);
    return DBS_OK;
}

inline dbs_status check_work(const char *fn, const void *d_work)
{
    if ((uintptr_t)d_work % 256) return dbs_fail(DBS_ERR_ARG, "%s: the workspace is not aligned to 256 bytes", fn);
    return DBS_OK;
}

inline dbs_status check_room(const char *fn, size_t need, const void *d_work, size_t work_bytes)
{
    if (need > work_bytes || (need && !d_work) || (uintptr_t)d_work % 256)
        return dbs_fail(DBS_ERR_ARG, "%s: needs %zu bytes of workspace at a multiple of 256, got %zu", fn, need, work_bytes);
    return DBS_OK;
}

#define CHECK(expr)                                    \
    do {                                               \
        const dbs_status st_ = (expr);                 \
        if (st_ != DBS_OK) return st_;                 \
    } while (0)

inline int64_t up8(int64_t n) { return (n + 7) / 8 * 8; }
inline size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// Parts of a caller's workspace, each at a multiple of 256 bytes.
struct Carve {
    uint8_t *base;
    size_t used = 0;
    void *take(size_t bytes)
    {
        void *p = base ? base + used : nullptr;
        used += up256(bytes);
        return p;
    }
};
