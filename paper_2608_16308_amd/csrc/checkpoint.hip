// 8-bit activation checkpoints and the elementwise part of the backward
// passes that reads them.
#include <algorithm>
#include <type_traits>

#include "device_common.hpp"
#include "layer.hpp"

namespace dbs {

// Chunks of eight columns, at any alignment: rows of odd lengths start
// anywhere.
template <class X> struct __attribute__((packed, aligned(2))) Vals8 {
    typename X::V8 v;
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
constexpr int CK_TPB = 256;
constexpr int CK_U = 2;      // chunks in flight per thread
constexpr int CK_CHUNK = 16; // columns of a chunk

// The chunks of a thread: from row to row in steps of the whole grid, with one
// division at the start.
struct Walk {
    int32_t row, chunk;
    __device__ Walk(uint32_t per, uint32_t first) : row((int32_t)(first / per)), chunk((int32_t)(first % per)) {}
    __device__ void step(const int32_t rows_on, const int32_t chunks_on, const int32_t per)
    {
        row += rows_on;
        chunk += chunks_on;
        if (chunk >= per) chunk -= per, ++row;
    }
};
// per: chunks of a row; rows_on, chunks_on: the grid's threads in rows and chunks
struct Grid {
    int32_t rows, cols, per, rows_on, chunks_on;
};

struct __attribute__((packed, aligned(1))) Codes16 {
    uint32_t w[4];
};
// A thread takes chunks of 16 columns, the two of a group in neighbouring
// lanes; a row's chunks are counted up to a whole group.
//
// Bound: by the bytes (2 in, 33/32 out per value).
template <class X>
__global__ __launch_bounds__(CK_TPB) void k_pack(const typename X::T *__restrict__ x, int64_t ldx, Grid g,
                                                 int8_t *__restrict__ codes, uint8_t *__restrict__ exps)
{
    const int64_t groups = g.per / 2;
    for (Walk at((uint32_t)g.per, blockIdx.x * CK_TPB + threadIdx.x); at.row < g.rows;) {
        float v[CK_U][16];
        int32_t row[CK_U], col[CK_U];
#pragma unroll
        for (int u = 0; u < CK_U; ++u, at.step(g.rows_on, g.chunks_on, g.per)) {
            row[u] = at.row, col[u] = CK_CHUNK * at.chunk;
            const int left = row[u] < g.rows ? g.cols - col[u] : 0;
            const typename X::T *p = x + (int64_t)row[u] * ldx + col[u];
            float lo[8], hi[8];
            load_vals<X>(p, left, lo);
            load_vals<X>(p + 8, left - 8, hi);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[u][k] = lo[k], v[u][8 + k] = hi[k];
        }
#pragma unroll
        for (int u = 0; u < CK_U; ++u) {
            float big = 0.f;
#pragma unroll
            for (int k = 0; k < 16; ++k) big = fmaxf(big, ck_mag(v[u][k]));
            big = fmaxf(big, __shfl_xor(big, 1, 64));
            const int left = g.cols - col[u];
            if (row[u] >= g.rows || left <= 0) continue;
            const int e = ck_exp<X>(big);
            if (col[u] % CK_GROUP == 0) exps[row[u] * groups + col[u] / CK_GROUP] = (uint8_t)(e + CK_BIAS);
            int8_t *dst = codes + (int64_t)row[u] * g.cols + col[u];
            Codes16 c = {{0u, 0u, 0u, 0u}};
#pragma unroll
            for (int k = 0; k < 16; ++k) c.w[k >> 2] |= (uint32_t)(ck_code(v[u][k], e) & 255) << (8 * (k & 3));
            if (left >= 16) *(Codes16 *)dst = c;
            else
#pragma unroll
                for (int k = 0; k < 16; ++k)
                    if (k < left) dst[k] = (int8_t)(c.w[k >> 2] >> (8 * (k & 3)));
        }
    }
}

// Chunks of eight columns here: a lane's 16 bytes lie beside its neighbours'.
template <class X>
__global__ __launch_bounds__(CK_TPB) void k_unpack(const int8_t *__restrict__ codes, const uint8_t *__restrict__ exps, Grid g,
                                                   typename X::T *__restrict__ y, int64_t ldy)
{
    constexpr int U = 2 * CK_U;
    const int64_t groups = (g.cols + CK_GROUP - 1) / CK_GROUP;
    for (Walk at((uint32_t)g.per, blockIdx.x * CK_TPB + threadIdx.x); at.row < g.rows;) {
        Codes8 c[U];
        int e[U];
        int32_t row[U], col[U];
#pragma unroll
        for (int u = 0; u < U; ++u, at.step(g.rows_on, g.chunks_on, g.per)) {
            row[u] = at.row, col[u] = 8 * at.chunk;
            if (row[u] >= g.rows) continue;
            c[u] = load_codes(codes + (int64_t)row[u] * g.cols + col[u], g.cols - col[u]);
            e[u] = (int)exps[row[u] * groups + col[u] / CK_GROUP] - CK_BIAS;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (row[u] >= g.rows) continue;
            float v[8];
            ck_values<X>(c[u], e[u], v);
            store_vals<X>(y + (int64_t)row[u] * ldy + col[u], g.cols - col[u], v);
        }
    }
}

// (bits only: one kernel for both types)
__global__ __launch_bounds__(CK_TPB) void k_align(const _Float16 *__restrict__ src, int64_t ld, Grid g, uint4 *__restrict__ dst,
                                                  int64_t ldd)
{
    for (Walk at((uint32_t)g.per, blockIdx.x * CK_TPB + threadIdx.x); at.row < g.rows;) {
        Fp16::V8 v[2 * CK_U];
        int32_t row[2 * CK_U], chunk[2 * CK_U];
#pragma unroll
        for (int u = 0; u < 2 * CK_U; ++u, at.step(g.rows_on, g.chunks_on, g.per)) {
            row[u] = at.row, chunk[u] = at.chunk;
            const _Float16 *p = src + (int64_t)min(row[u], g.rows - 1) * ld;
            if (g.cols >= 8) v[u] = load_end<Fp16>(p, 8 * chunk[u], g.cols);
            else
#pragma unroll
                for (int k = 0; k < 8; ++k) v[u][k] = k < g.cols ? p[min(k, g.cols - 1)] : (_Float16)0.f;
        }
#pragma unroll
        for (int u = 0; u < 2 * CK_U; ++u)
            if (row[u] < g.rows) dst[(int64_t)row[u] * (ldd / 8) + chunk[u]] = __builtin_bit_cast(uint4, v[u]);
    }
}

constexpr int SL_WAVES = 4;                // waves of a workgroup, each a row at a time
constexpr int SL_COLS = 64 * 8;            // columns of a workgroup
constexpr int SUM_WAVES = 16;
static_assert(SL_WAVES == 4, "the maxima of four waves");

__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, WAVE));
    return v;
}

// Eight columns of a row of the activation gradients in 32 bits, the chunk `col`
// (`left` columns up to the row's end, zeros behind it).
template <class X, bool GATED>
__device__ __forceinline__ void slope_chunk(const SlopeArgs &a, int row, int col, int left, float (&dz)[8], float (&du)[8])
{
    typedef typename X::T T;
    const int64_t groups = (a.cols + CK_GROUP - 1) / CK_GROUP;
    auto held = [&](const HeldIn &h, float (&v)[8]) {
        if (h.codes) ck_values<X>(load_codes(h.codes + (int64_t)row * a.cols + col, left),
                                (int)h.exps[row * groups + col / CK_GROUP] - CK_BIAS, v);
        else load_vals<X>((const T *)h.full + (int64_t)row * h.ld + col, left, v);
    };
    float dy[8], z[8], up[8], f[8], d[8];
    load_vals<X>((const T *)a.dy + (int64_t)row * a.lddy + col, left, dy);
    if (a.pre.codes || a.pre.full) held(a.pre, z);
    else
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = 0.f;
    if (GATED) held(a.up, up);
    act_slopes(a.act, z, f, d);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (GATED) du[i] = i < left ? dy[i] * f[i] : 0.f;
        dz[i] = i < left ? (GATED ? dy[i] * up[i] : dy[i]) * d[i] : 0.f;
    }
}
// The rows of workgroups along the rows.
__device__ __forceinline__ int slope_row(const SlopeArgs &a, int block) { return (int)((int64_t)a.rows * block / a.row_blocks); }

// The sums of the columns are added in a fixed order: a lane's rows, the
// waves, then the workgroups along the rows (k_slope_sum).
template <class X, bool GATED>
__global__ __launch_bounds__(64 * SL_WAVES) void k_slope(SlopeArgs a)
{
    typedef typename X::T T;
    constexpr bool RANGE = std::is_same<X, Fp16>::value;
    __shared__ float part[SL_WAVES][SL_COLS];
    const int lane = lane_id(), wave = wave_id();
    const int col = (int)blockIdx.x * SL_COLS + 8 * lane, left = a.cols - col;
    const int r1 = slope_row(a, (int)blockIdx.y + 1);
    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, most = 0.f;
    if (left > 0)
        for (int row = slope_row(a, (int)blockIdx.y) + wave; row < r1; row += SL_WAVES) {
            float dz[8], du[8];
            slope_chunk<X, GATED>(a, row, col, left, dz, du);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += dz[i];
            if (RANGE && a.most)
#pragma unroll
                for (int i = 0; i < 8; ++i) most = fmaxf(most, GATED ? fmaxf(ck_mag(dz[i]), ck_mag(du[i])) : ck_mag(dz[i]));
            if (a.dz) {
                store_vals<X>((T *)a.dz + (int64_t)row * a.ldz + col, 8, dz);
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
        __syncthreads();
    }
    if (RANGE && a.most) {
        most = wave_max(most);
        if (lane == 0) part[wave][0] = most;
        __syncthreads();
        if (threadIdx.x == 0)
            a.most[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = fmaxf(fmaxf(part[0][0], part[1][0]), fmaxf(part[2][0], part[3][0]));
    }
}

// fp16: where the largest dz or du has left the type's range, all of them again,
// times 2^-s.  Nearly always there is nothing to do beside reading the workgroups'
// maxima (4 us of a call; no atomics and no answer on the host, so that a captured
// call follows its inputs).
template <bool GATED> __global__ __launch_bounds__(64 * SL_WAVES) void k_slope_range(SlopeArgs a, int32_t strips)
{
    __shared__ float part[SL_WAVES];
    const int lane = lane_id(), wave = wave_id();
    const int64_t n = (int64_t)strips * a.row_blocks;
    float most = 0.f;
    for (int64_t i = threadIdx.x; i < n; i += 64 * SL_WAVES) most = fmaxf(most, a.most[i]);
    most = wave_max(most);
    if (lane == 0) part[wave] = most;
    __syncthreads();
    const int s = slope_exp(fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3])));
    if (blockIdx.x == 0 && threadIdx.x == 0) a.most[n] = __builtin_amdgcn_ldexpf(1.f, s);
    if (s == 0) return;
    const float by = __builtin_amdgcn_ldexpf(1.f, -s);
    for (int64_t at = blockIdx.x; at < n; at += gridDim.x) {
        const int block = (int)(at / strips), col = (int)(at % strips) * SL_COLS + 8 * lane, left = a.cols - col;
        const int r1 = slope_row(a, block + 1);
        if (left <= 0) continue;
        for (int row = slope_row(a, block) + wave; row < r1; row += SL_WAVES) {
            float dz[8], du[8];
            slope_chunk<Fp16, GATED>(a, row, col, left, dz, du);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                dz[i] *= by;
                if (GATED) du[i] *= by;
            }
            store_vals<Fp16>((_Float16 *)a.dz + (int64_t)row * a.ldz + col, 8, dz);
            if (GATED) store_vals<Fp16>((_Float16 *)a.du + (int64_t)row * a.ldz + col, 8, du);
        }
    }
}

// The workgroups' sums, a column a lane, the rows shared out to the waves.
template <class X>
__global__ __launch_bounds__(64 * SUM_WAVES) void k_slope_sum(const float *__restrict__ sums, int32_t n, int32_t cols,
                                                              typename X::T *__restrict__ db, int32_t first)
{
    __shared__ float part[SUM_WAVES][64];
    const int lane = lane_id(), wave = wave_id(), c = ((int)blockIdx.x + first) * 64 + lane;
    float s = 0.f;
    if (c < cols)
#pragma unroll 4
        for (int i = wave; i < n; i += SUM_WAVES) s += sums[i * (int64_t)cols + c];
    part[wave][lane] = s;
    __syncthreads();
    if (wave != 0 || c >= cols) return;
#pragma unroll
    for (int w = 1; w < SUM_WAVES; ++w) s += part[w][lane];
    db[c] = (typename X::T)s;
}

// A grid over rows of `per` chunks: a thread per chunk, or as many as are
// resident at once.
static Grid chunk_grid(int32_t rows, int32_t cols, int32_t per, int32_t cus, unsigned *blocks)
{
    const uint64_t chunks = (uint64_t)rows * per;
    *blocks = (unsigned)std::max<uint64_t>(1, std::min<uint64_t>((chunks + CK_TPB - 1) / CK_TPB, (uint64_t)cus * 8));
    const uint32_t threads = *blocks * CK_TPB;
    return Grid{rows, cols, per, (int32_t)(threads / (uint32_t)per), (int32_t)(threads % (uint32_t)per)};
}

hipError_t launch_pack(bool bf16, const void *x, int64_t ldx, int32_t rows, int32_t cols, int8_t *codes, uint8_t *exps,
                       int32_t cus, hipStream_t s)
{
    if (rows == 0 || cols == 0) return hipSuccess;
    unsigned n;
    const Grid g = chunk_grid(rows, cols, 2 * ((cols + CK_GROUP - 1) / CK_GROUP), cus, &n);
    if (bf16) hipLaunchKernelGGL(k_pack<Bf16>, dim3(n), dim3(CK_TPB), 0, s, (const Bf16::T *)x, ldx, g, codes, exps);
    else hipLaunchKernelGGL(k_pack<Fp16>, dim3(n), dim3(CK_TPB), 0, s, (const Fp16::T *)x, ldx, g, codes, exps);
    return hipGetLastError();
}

hipError_t launch_unpack(bool bf16, const int8_t *codes, const uint8_t *exps, int32_t rows, int32_t cols, void *y,
                         int64_t ldy, int32_t cus, hipStream_t s)
{
    if (rows == 0 || cols == 0) return hipSuccess;
    unsigned n;
    const Grid g = chunk_grid(rows, cols, (cols + 7) / 8, cus, &n);
    if (bf16) hipLaunchKernelGGL(k_unpack<Bf16>, dim3(n), dim3(CK_TPB), 0, s, codes, exps, g, (Bf16::T *)y, ldy);
    else hipLaunchKernelGGL(k_unpack<Fp16>, dim3(n), dim3(CK_TPB), 0, s, codes, exps, g, (Fp16::T *)y, ldy);
    return hipGetLastError();
}

hipError_t launch_align(const void *src, int64_t ld, int32_t rows, int32_t cols, void *dst, int64_t ldd, int32_t cus,
                        hipStream_t s)
{
    if (rows == 0 || cols == 0) return hipSuccess;
    unsigned n;
    const Grid g = chunk_grid(rows, cols, (cols + 7) / 8, cus, &n);
    hipLaunchKernelGGL(k_align, dim3(n), dim3(CK_TPB), 0, s, (const _Float16 *)src, ld, g, (uint4 *)dst, ldd);
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

int64_t slope_blocks(int32_t rows, int32_t cols, int32_t cus)
{
    return (((int64_t)cols + SL_COLS - 1) / SL_COLS) * slope_row_blocks(rows, cols, cus);
}

template <class X> static hipError_t slope_t(bool gated, const SlopeArgs &a, hipStream_t s)
{
    const dim3 grid((unsigned)((a.cols + SL_COLS - 1) / SL_COLS), (unsigned)a.row_blocks), block(64 * SL_WAVES);
    if (gated) hipLaunchKernelGGL((k_slope<X, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((k_slope<X, false>), grid, block, 0, s, a);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && a.most) {
        const unsigned n = std::min(grid.x * grid.y, 1024u);
        if (gated) hipLaunchKernelGGL(k_slope_range<true>, dim3(n), block, 0, s, a, (int32_t)grid.x);
        else hipLaunchKernelGGL(k_slope_range<false>, dim3(n), block, 0, s, a, (int32_t)grid.x);
        e = hipGetLastError();
    }
    if (e == hipSuccess && a.sums) {
        e = launch_parts(((int64_t)a.cols + 63) / 64, 64 * SUM_WAVES, [&](int32_t first, dim3 n) {
            hipLaunchKernelGGL(k_slope_sum<X>, n, dim3(64 * SUM_WAVES), 0, s, a.sums, a.row_blocks, a.cols,
                               (typename X::T *)a.db, first);
        });
    }
    return e;
}
hipError_t launch_slope(bool bf16, bool gated, const SlopeArgs &a, hipStream_t s)
{
    if (a.cols == 0) return hipSuccess;
    return bf16 ? slope_t<Bf16>(gated, a, s) : slope_t<Fp16>(gated, a, s);
}

}  // namespace dbs
