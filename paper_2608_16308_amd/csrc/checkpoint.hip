// 8-bit activation checkpoints and the elementwise part of the backward
// passes that reads them.
#include <algorithm>

#include "device_common.hpp"
#include "layer.hpp"

namespace dbs {

// Chunks of eight columns, at any alignment: rows of odd lengths start
// anywhere.
template <class X> struct __attribute__((packed, aligned(2))) Vals8 {
    typename X::V8 v;
};
struct __attribute__((packed, aligned(1))) Codes8 {
    uint32_t w[2];
};

template <class X>
__device__ __forceinline__ void load_vals(const typename X::T *p, int left, float (&v)[8])
{
    if (left >= 8) {
        const typename X::V8 t = ((const Vals8<X> *)p)->v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)t[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < left ? (float)p[i] : 0.f;
    }
}
template <class X>
__device__ __forceinline__ void store_vals(typename X::T *p, int left, const float (&v)[8])
{
    typename X::V8 t;
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = (typename X::T)v[i];
    if (left >= 8) ((Vals8<X> *)p)->v = t;
    else
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) p[i] = t[i];
}
__device__ __forceinline__ Codes8 load_codes(const int8_t *p, int left)
{
    if (left >= 8) return *(const Codes8 *)p;
    Codes8 c = {{0u, 0u}};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < left) c.w[i >> 2] |= (uint32_t)(uint8_t)p[i] << (8 * (i & 3));
    return c;
}
template <class X> __device__ __forceinline__ void decode8(Codes8 c, int e, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = ck_value<X>((int)(int8_t)(c.w[i >> 2] >> (8 * (i & 3))), e);
}

constexpr int CK_TPB = 256;
constexpr int CK_U = 4;  // chunks in flight per thread

// A thread takes chunks of eight columns, the four of a group in neighbouring
// lanes; a row's chunks are counted up to a whole group.
template <class X>
__global__ __launch_bounds__(CK_TPB) void k_pack(const typename X::T *__restrict__ x, int64_t ldx, int32_t rows,
                                                 int32_t cols, int8_t *__restrict__ codes, uint8_t *__restrict__ exps)
{
    const uint32_t groups = (uint32_t)((cols + CK_GROUP - 1) / CK_GROUP), per = 4 * groups;
    const uint64_t total = (uint64_t)rows * per, stride = (uint64_t)gridDim.x * CK_TPB;
    for (uint64_t i0 = (uint64_t)blockIdx.x * CK_TPB + threadIdx.x; i0 < total; i0 += CK_U * stride) {
        float v[CK_U][8];
        int32_t row[CK_U], col[CK_U];
#pragma unroll
        for (int u = 0; u < CK_U; ++u) {
            const uint64_t i = i0 + u * stride;
            row[u] = i < total ? (int32_t)(i / per) : -1;
            col[u] = 8 * (int32_t)(i - (uint64_t)(uint32_t)row[u] * per);
            load_vals<X>(x + (int64_t)row[u] * ldx + col[u], row[u] < 0 ? 0 : cols - col[u], v[u]);
        }
#pragma unroll
        for (int u = 0; u < CK_U; ++u) {
            float big = 0.f;
#pragma unroll
            for (int k = 0; k < 8; ++k) big = fmaxf(big, ck_mag(v[u][k]));
            big = fmaxf(big, __shfl_xor(big, 1, 64));
            big = fmaxf(big, __shfl_xor(big, 2, 64));
            if (row[u] < 0 || col[u] >= cols) continue;
            const int e = ck_exp<X>(big);
            if (col[u] % CK_GROUP == 0) exps[(int64_t)row[u] * groups + col[u] / CK_GROUP] = (uint8_t)(e + CK_BIAS);
            int8_t *dst = codes + (int64_t)row[u] * cols + col[u];
            Codes8 c = {{0u, 0u}};
#pragma unroll
            for (int k = 0; k < 8; ++k) c.w[k >> 2] |= (uint32_t)(ck_code(v[u][k], e) & 255) << (8 * (k & 3));
            const int left = cols - col[u];
            if (left >= 8) *(Codes8 *)dst = c;
            else
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (k < left) dst[k] = (int8_t)(c.w[k >> 2] >> (8 * (k & 3)));
        }
    }
}

template <class X>
__global__ __launch_bounds__(CK_TPB) void k_unpack(const int8_t *__restrict__ codes, const uint8_t *__restrict__ exps,
                                                   int32_t rows, int32_t cols, typename X::T *__restrict__ y,
                                                   int64_t ldy)
{
    const uint32_t groups = (uint32_t)((cols + CK_GROUP - 1) / CK_GROUP), per = (uint32_t)((cols + 7) / 8);
    const uint64_t total = (uint64_t)rows * per, stride = (uint64_t)gridDim.x * CK_TPB;
    for (uint64_t i0 = (uint64_t)blockIdx.x * CK_TPB + threadIdx.x; i0 < total; i0 += CK_U * stride) {
        Codes8 c[CK_U];
        int e[CK_U];
        int32_t row[CK_U], col[CK_U];
#pragma unroll
        for (int u = 0; u < CK_U; ++u) {
            const uint64_t i = i0 + u * stride;
            row[u] = i < total ? (int32_t)(i / per) : -1;
            col[u] = 8 * (int32_t)(i - (uint64_t)(uint32_t)row[u] * per);
            if (row[u] < 0) continue;
            c[u] = load_codes(codes + (int64_t)row[u] * cols + col[u], cols - col[u]);
            e[u] = (int)exps[(int64_t)row[u] * groups + col[u] / CK_GROUP] - CK_BIAS;
        }
#pragma unroll
        for (int u = 0; u < CK_U; ++u) {
            if (row[u] < 0) continue;
            float v[8];
            decode8<X>(c[u], e[u], v);
            store_vals<X>(y + (int64_t)row[u] * ldy + col[u], cols - col[u], v);
        }
    }
}

// (bits only: one kernel for both types)
__global__ __launch_bounds__(CK_TPB) void k_align(const _Float16 *__restrict__ src, int64_t ld, int32_t rows, int32_t cols,
                                                  uint4 *__restrict__ dst, int64_t ldd)
{
    const uint32_t per = (uint32_t)((cols + 7) / 8);
    const uint64_t total = (uint64_t)rows * per, stride = (uint64_t)gridDim.x * CK_TPB;
    for (uint64_t i0 = (uint64_t)blockIdx.x * CK_TPB + threadIdx.x; i0 < total; i0 += CK_U * stride) {
        Fp16::V8 v[CK_U];
        int64_t at[CK_U];
#pragma unroll
        for (int u = 0; u < CK_U; ++u) {
            const uint64_t i = i0 + u * stride < total ? i0 + u * stride : total - 1;
            const int32_t row = (int32_t)(i / per), col = 8 * (int32_t)(i - (uint64_t)row * per);
            const _Float16 *p = src + (int64_t)row * ld;
            if (cols >= 8) v[u] = load_end<Fp16>(p, col, cols);
            else
#pragma unroll
                for (int k = 0; k < 8; ++k) v[u][k] = k < cols ? p[min(k, cols - 1)] : (_Float16)0.f;
            at[u] = ((int64_t)row * ldd + col) / 8;
        }
#pragma unroll
        for (int u = 0; u < CK_U; ++u)
            if (i0 + u * stride < total) dst[at[u]] = __builtin_bit_cast(uint4, v[u]);
    }
}

constexpr int SL_WAVES = 4;                // waves of a workgroup, each a row at a time
constexpr int SL_COLS = 64 * 8;            // columns of a workgroup

// The sums of the columns are added in a fixed order: a lane's rows, the
// waves, then the workgroups along the rows (k_slope_sum).
template <class X, bool GATED>
__global__ __launch_bounds__(64 * SL_WAVES) void k_slope(SlopeArgs a)
{
    typedef typename X::T T;
    __shared__ float part[SL_WAVES][SL_COLS];
    const int lane = lane_id(), wave = wave_id();
    const int col = (int)blockIdx.x * SL_COLS + 8 * lane, left = a.cols - col;
    const int r0 = (int)((int64_t)a.rows * blockIdx.y / a.row_blocks);
    const int r1 = (int)((int64_t)a.rows * (blockIdx.y + 1) / a.row_blocks);
    const int64_t groups = (a.cols + CK_GROUP - 1) / CK_GROUP;
    auto held = [&](const HeldIn &h, int row, float (&v)[8]) {
        if (h.codes) decode8<X>(load_codes(h.codes + (int64_t)row * a.cols + col, left),
                                (int)h.exps[row * groups + col / CK_GROUP] - CK_BIAS, v);
        else load_vals<X>((const T *)h.full + (int64_t)row * h.ld + col, left, v);
    };
    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (left > 0)
        for (int row = r0 + wave; row < r1; row += SL_WAVES) {
            float dy[8], z[8], up[8], du[8];
            load_vals<X>((const T *)a.dy + (int64_t)row * a.lddy + col, left, dy);
            if (a.pre.codes || a.pre.full) held(a.pre, row, z);
            else
#pragma unroll
                for (int i = 0; i < 8; ++i) z[i] = 0.f;
            if (GATED) held(a.up, row, up);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float f;
                const float d = act_slope(a.act, z[i], f);
                if (GATED) du[i] = dy[i] * f;
                // (columns past the last: the zeros that fill the row)
                z[i] = i < left ? (GATED ? dy[i] * up[i] * d : dy[i] * d) : 0.f;
                if (GATED && i >= left) du[i] = 0.f;
                sum[i] += z[i];
            }
            if (a.dz) {
                store_vals<X>((T *)a.dz + (int64_t)row * a.ldz + col, 8, z);
                if (GATED) store_vals<X>((T *)a.du + (int64_t)row * a.ldz + col, 8, du);
            }
        }
    if (!GATED && a.sums) {
#pragma unroll
        for (int i = 0; i < 8; ++i) part[wave][8 * lane + i] = sum[i];
        __syncthreads();
        for (int c = (int)threadIdx.x; c < SL_COLS; c += 64 * SL_WAVES) {
            const int64_t at = (int64_t)blockIdx.x * SL_COLS + c;
            if (at >= a.cols) continue;
            float s = 0.f;
#pragma unroll
            for (int w = 0; w < SL_WAVES; ++w) s += part[w][c];
            a.sums[blockIdx.y * (int64_t)a.cols + at] = s;
        }
    }
}

template <class X>
__global__ __launch_bounds__(256) void k_slope_sum(const float *__restrict__ sums, int32_t n, int32_t cols,
                                                   typename X::T *__restrict__ db)
{
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (c >= cols) return;
    float s = 0.f;
    for (int i = 0; i < n; ++i) s += sums[i * (int64_t)cols + c];
    db[c] = (typename X::T)s;
}

static unsigned chunk_grid(uint64_t chunks, int32_t cus)
{
    return (unsigned)std::min<uint64_t>((chunks + CK_TPB - 1) / CK_TPB, (uint64_t)cus * 8);
}

template <class X>
static hipError_t pack_t(const void *x, int64_t ldx, int32_t rows, int32_t cols, int8_t *codes, uint8_t *exps, int32_t cus,
                         hipStream_t s)
{
    const uint64_t chunks = (uint64_t)rows * 4 * ((cols + CK_GROUP - 1) / CK_GROUP);
    hipLaunchKernelGGL(k_pack<X>, dim3(chunk_grid(chunks, cus)), dim3(CK_TPB), 0, s, (const typename X::T *)x, ldx, rows,
                       cols, codes, exps);
    return hipGetLastError();
}
hipError_t launch_pack(bool bf16, const void *x, int64_t ldx, int32_t rows, int32_t cols, int8_t *codes, uint8_t *exps,
                       int32_t cus, hipStream_t s)
{
    if (rows == 0 || cols == 0) return hipSuccess;
    return bf16 ? pack_t<Bf16>(x, ldx, rows, cols, codes, exps, cus, s) : pack_t<Fp16>(x, ldx, rows, cols, codes, exps, cus, s);
}

template <class X>
static hipError_t unpack_t(const int8_t *codes, const uint8_t *exps, int32_t rows, int32_t cols, void *y, int64_t ldy,
                           int32_t cus, hipStream_t s)
{
    const uint64_t chunks = (uint64_t)rows * ((cols + 7) / 8);
    hipLaunchKernelGGL(k_unpack<X>, dim3(chunk_grid(chunks, cus)), dim3(CK_TPB), 0, s, codes, exps, rows, cols,
                       (typename X::T *)y, ldy);
    return hipGetLastError();
}
hipError_t launch_unpack(bool bf16, const int8_t *codes, const uint8_t *exps, int32_t rows, int32_t cols, void *y,
                         int64_t ldy, int32_t cus, hipStream_t s)
{
    if (rows == 0 || cols == 0) return hipSuccess;
    return bf16 ? unpack_t<Bf16>(codes, exps, rows, cols, y, ldy, cus, s) : unpack_t<Fp16>(codes, exps, rows, cols, y, ldy, cus, s);
}

hipError_t launch_align(const void *src, int64_t ld, int32_t rows, int32_t cols, void *dst, int64_t ldd, int32_t cus,
                        hipStream_t s)
{
    if (rows == 0 || cols == 0) return hipSuccess;
    const uint64_t chunks = (uint64_t)rows * ((cols + 7) / 8);
    hipLaunchKernelGGL(k_align, dim3(chunk_grid(chunks, cus)), dim3(CK_TPB), 0, s, (const _Float16 *)src, ld, rows, cols,
                       (uint4 *)dst, ldd);
    return hipGetLastError();
}

// Workgroups along the rows: enough to fill the device, none with less than
// a row for each wave.
int32_t slope_row_blocks(int32_t rows, int32_t cols, int32_t cus)
{
    const int64_t strips = (cols + SL_COLS - 1) / SL_COLS;
    const int64_t want = strips ? (8 * (int64_t)cus + strips - 1) / strips : 1;
    return (int32_t)std::max<int64_t>(1, std::min<int64_t>({want, (rows + SL_WAVES - 1) / SL_WAVES, 65535}));
}

template <class X> static hipError_t slope_t(bool gated, const SlopeArgs &a, hipStream_t s)
{
    const dim3 grid((unsigned)((a.cols + SL_COLS - 1) / SL_COLS), (unsigned)a.row_blocks), block(64 * SL_WAVES);
    if (gated) hipLaunchKernelGGL((k_slope<X, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((k_slope<X, false>), grid, block, 0, s, a);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && a.sums) {
        hipLaunchKernelGGL(k_slope_sum<X>, dim3((unsigned)((a.cols + 255) / 256)), dim3(256), 0, s, a.sums, a.row_blocks,
                           a.cols, (typename X::T *)a.db);
        e = hipGetLastError();
    }
    return e;
}
hipError_t launch_slope(bool bf16, bool gated, const SlopeArgs &a, hipStream_t s)
{
    if (a.cols == 0) return hipSuccess;
    return bf16 ? slope_t<Bf16>(gated, a, s) : slope_t<Fp16>(gated, a, s);
}

}  // namespace dbs
