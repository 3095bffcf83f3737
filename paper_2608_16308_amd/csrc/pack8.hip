// 16-bit matrices into blocks of 8-bit floating point and back.
#include <algorithm>

#include "device_common.hpp"
#include "float8.hpp"

namespace dbs {

constexpr int P8_TPB = 256;
constexpr int P8_LINE = E8_BLOCK + 16;  // bytes of a turned row in LDS

__device__ __forceinline__ float max16(float v)
{
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    return v;
}
// Bytes behind the last block's exponent.
__device__ __forceinline__ void pad_exps(const Blocks &b, int64_t row, int64_t blocks)
{
    for (int64_t i = blocks; i < b.lde; ++i) b.exps[row * b.lde + i] = E8_BIAS;
}

// A workgroup takes a tile of 128 x 128, a thread 8 rows of 8 columns of it: the
// 16 lanes beside each other have a row's block, the 16 groups of them a column's.
// Turned codes change places in LDS, so that both results are written in whole
// lines of 128 bytes.  Bound by the bytes.
template <class X, bool CODES> __global__ __launch_bounds__(P8_TPB) void k_pack8(Pack8Args a)
{
    typedef typename X::T T;
    __shared__ float most[4][E8_BLOCK], sums[4][E8_BLOCK];
    __shared__ __attribute__((aligned(16))) uint8_t lines[E8_BLOCK * P8_LINE];
    const int lane = lane_id(), wave = wave_id(), rg = (int)threadIdx.x >> 4, cc = (int)threadIdx.x & 15;
    const int64_t tile = (int64_t)blockIdx.x + a.first;
    const int tr = (int)(tile / a.tiles_c), tc = (int)(tile % a.tiles_c);
    const int row0 = tr * E8_BLOCK + 8 * rg, col0 = tc * E8_BLOCK + 8 * cc, left = a.cols - col0;

    float v[8][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int64_t row = row0 + i;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
        if (row >= a.rows || left <= 0) continue;
        if constexpr (CODES) {
            e8_values<X>(*(const uint2 *)(a.from.codes + row * a.from.ld + col0), (int)a.from.exps[row * a.from.lde + tc] - E8_BIAS, v[i]);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = j < left ? (float)(T)v[i][j] : 0.f;
        } else {
            const T *p = (const T *)a.x + row * a.ldx + col0;
            if (left >= 8) {
                const typename X::V8 t = load_eight<X>(p);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] = (float)t[j];
            } else
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < left) v[i][j] = (float)p[j];
        }
    }
    // largest magnitudes of the thread's rows and columns
    float mr[8], mc[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) mr[i] = mc[i] = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float m = ck_mag(v[i][j]);
            mr[i] = fmaxf(mr[i], m), mc[j] = fmaxf(mc[j], m);
        }
    if (a.tile || a.turned.codes || a.sums) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float m = mc[j], s = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) s += v[i][j];
            m = fmaxf(m, __shfl_xor(m, 16, 64)), s += __shfl_xor(s, 16, 64);
            m = fmaxf(m, __shfl_xor(m, 32, 64)), s += __shfl_xor(s, 32, 64);
            if (lane < 16) most[wave][8 * cc + j] = m, sums[wave][8 * cc + j] = s;
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 8; ++j)
            mc[j] = fmaxf(fmaxf(most[0][8 * cc + j], most[1][8 * cc + j]), fmaxf(most[2][8 * cc + j], most[3][8 * cc + j]));
    }
    if (a.tile) {
        float m = mc[0];
#pragma unroll
        for (int j = 1; j < 8; ++j) m = fmaxf(m, mc[j]);
        m = max16(m);
#pragma unroll
        for (int i = 0; i < 8; ++i) mr[i] = mc[i] = m;
    }
    if (a.sums && threadIdx.x < E8_BLOCK) {
        const int c = (int)threadIdx.x, col = tc * E8_BLOCK + c;
        if (col < a.cols) a.sums[tr * (int64_t)a.cols + col] = sums[0][c] + sums[1][c] + sums[2][c] + sums[3][c];
    }
    if (a.to.codes) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t row = row0 + i;
            const int e = e8_exp(a.tile ? mr[i] : max16(mr[i]));
            if (row >= a.rows) continue;
            *(uint2 *)(a.to.codes + row * a.to.ld + col0) = e8_codes(v[i], e);
            if (cc == 0 && (!a.tile || (rg == 0 && i == 0))) {
                const int64_t at = row >> a.to.shift;
                a.to.exps[at * a.to.lde + tc] = (uint8_t)(e + E8_BIAS);
                if (tc == a.tiles_c - 1) pad_exps(a.to, at, a.tiles_c);
            }
        }
    }
    if (a.turned.codes) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float t[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) t[i] = v[i][j];
            const int e = e8_exp(mc[j]);
            *(uint2 *)(lines + (8 * cc + j) * P8_LINE + 8 * rg) = e8_codes(t, e);
            if (rg == 0 && j < left && (!a.tile || (cc == 0 && j == 0))) {
                const int64_t at = (int64_t)(col0 + j) >> a.turned.shift, blocks = e8_blocks(a.rows);
                a.turned.exps[at * a.turned.lde + tr] = (uint8_t)(e + E8_BIAS);
                if (tr == blocks - 1) pad_exps(a.turned, at, blocks);
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = i * P8_TPB + (int)threadIdx.x, line = c >> 3, at = 16 * (c & 7);
            const int64_t col = (int64_t)tc * E8_BLOCK + line;
            if (col < a.cols) *(uint4 *)(a.turned.codes + col * a.turned.ld + (int64_t)tr * E8_BLOCK + at) = *(const uint4 *)(lines + line * P8_LINE + at);
        }
    }
}

// A thread per chunk of eight columns.
template <class X>
__global__ __launch_bounds__(P8_TPB) void k_unpack8(Blocks b, int32_t rows, int32_t cols, int32_t per, typename X::T *y, int64_t ldy)
{
    const int64_t chunks = (int64_t)rows * per;
    for (int64_t c = (int64_t)blockIdx.x * P8_TPB + threadIdx.x; c < chunks; c += (int64_t)gridDim.x * P8_TPB) {
        const int64_t row = c / per;
        const int col = 8 * (int)(c - row * per), left = cols - col;
        float v[8];
        e8_values<X>(*(const uint2 *)(b.codes + row * b.ld + col), (int)b.exps[(row >> b.shift) * b.lde + col / E8_BLOCK] - E8_BIAS, v);
        typename X::T *p = y + row * ldy + col;
        typename X::V8 t;
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = (typename X::T)v[i];
        if (left >= 8) ((Eight<X> *)p)->v = t;
        else
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < left) p[i] = t[i];
    }
}

// A tile of codes a workgroup, turned in LDS; its exponent goes with it.
__global__ __launch_bounds__(P8_TPB) void k_turn8(Blocks b, int32_t rows, int32_t cols, int32_t tiles_c, int32_t first, Blocks to)
{
    __shared__ __attribute__((aligned(16))) uint8_t lines[E8_BLOCK * P8_LINE];
    const int64_t tile = (int64_t)blockIdx.x + first;
    const int tr = (int)(tile / tiles_c), tc = (int)(tile % tiles_c);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = i * P8_TPB + (int)threadIdx.x, line = c >> 3, at = 16 * (c & 7);
        const int64_t row = (int64_t)tr * E8_BLOCK + line;
        uint4 v = {0, 0, 0, 0};
        if (row < rows) v = *(const uint4 *)(b.codes + row * b.ld + (int64_t)tc * E8_BLOCK + at);
        *(uint4 *)(lines + line * P8_LINE + at) = v;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = i * P8_TPB + (int)threadIdx.x, line = c >> 3, at = 16 * (c & 7);
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < 16; ++k) w[k >> 2] |= (uint32_t)lines[(at + k) * P8_LINE + line] << (8 * (k & 3));
        const int64_t col = (int64_t)tc * E8_BLOCK + line;
        if (col < cols) *(uint4 *)(to.codes + col * to.ld + (int64_t)tr * E8_BLOCK + at) = uint4{w[0], w[1], w[2], w[3]};
    }
    if (threadIdx.x == 0) {
        to.exps[(int64_t)tc * to.lde + tr] = b.exps[(int64_t)tr * b.lde + tc];
        const int64_t blocks = e8_blocks(rows);
        if (tr == blocks - 1) pad_exps(to, tc, blocks);
    }
}

constexpr int64_t MAX_TILES8 = 1 << 30;

hipError_t launch_pack8(bool bf16, Pack8Args a, hipStream_t s)
{
    if (a.rows == 0 || a.cols == 0) return hipSuccess;
    const int64_t tiles = e8_blocks(a.rows) * e8_blocks(a.cols);
    if (tiles > MAX_TILES8) return hipErrorInvalidConfiguration;
    a.tiles_c = (int32_t)e8_blocks(a.cols);
    return launch_parts(tiles, P8_TPB, [&](int32_t first, dim3 grid) {
        a.first = first;
        if (a.from.codes) {
            if (bf16) hipLaunchKernelGGL((k_pack8<Bf16, true>), grid, dim3(P8_TPB), 0, s, a);
            else hipLaunchKernelGGL((k_pack8<Fp16, true>), grid, dim3(P8_TPB), 0, s, a);
        } else if (bf16) hipLaunchKernelGGL((k_pack8<Bf16, false>), grid, dim3(P8_TPB), 0, s, a);
        else hipLaunchKernelGGL((k_pack8<Fp16, false>), grid, dim3(P8_TPB), 0, s, a);
    });
}

hipError_t launch_unpack8(bool bf16, const Blocks &b, int32_t rows, int32_t cols, void *y, int64_t ldy, int32_t cus, hipStream_t s)
{
    if (rows == 0 || cols == 0) return hipSuccess;
    const int32_t per = (cols + 7) / 8;
    const dim3 grid((unsigned)std::min<int64_t>(((int64_t)rows * per + P8_TPB - 1) / P8_TPB, 16 * (int64_t)cus)), block(P8_TPB);
    if (bf16) hipLaunchKernelGGL(k_unpack8<Bf16>, grid, block, 0, s, b, rows, cols, per, (Bf16::T *)y, ldy);
    else hipLaunchKernelGGL(k_unpack8<Fp16>, grid, block, 0, s, b, rows, cols, per, (Fp16::T *)y, ldy);
    return hipGetLastError();
}

hipError_t launch_turn8(const Blocks &b, int32_t rows, int32_t cols, const Blocks &to, hipStream_t s)
{
    if (rows == 0 || cols == 0) return hipSuccess;
    const int64_t tiles = e8_blocks(rows) * e8_blocks(cols);
    if (tiles > MAX_TILES8) return hipErrorInvalidConfiguration;
    return launch_parts(tiles, P8_TPB, [&](int32_t first, dim3 grid) {
        hipLaunchKernelGGL(k_turn8, grid, dim3(P8_TPB), 0, s, b, rows, cols, (int32_t)e8_blocks(cols), first, to);
    });
}

}  // namespace dbs
