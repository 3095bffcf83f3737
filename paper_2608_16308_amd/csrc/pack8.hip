// 16-bit matrices into blocks of 8-bit floating point and back.
#include <algorithm>
#include <type_traits>

#include "device_common.hpp"
#include "float8.hpp"

namespace dbs {

constexpr int P8_TPB = 256;

// Bytes behind the last block's exponent.
__device__ __forceinline__ void pad_exps(const Blocks &b, int64_t row, int64_t blocks)
{
    for (int64_t i = blocks; i < b.lde; ++i) b.exps[row * b.lde + i] = E8_BIAS;
}

// Row blocks alone: eight columns a lane, 16 lanes a block, P8_U chunks in flight.
// Bound by the bytes (4096x4096 in bf16: 13.4 us, 3.8 TB/s).
constexpr int P8_U = 4;
template <class X> __global__ __launch_bounds__(P8_TPB) void k_pack8_rows(Pack8Args a)
{
    typedef typename X::T T;
    const int per = (int)e8_blocks(a.cols) * 16;  // chunks of a row
    const int64_t all = (int64_t)a.rows * per, stride = (int64_t)gridDim.x * P8_TPB;
    for (int64_t c0 = (int64_t)blockIdx.x * P8_TPB + threadIdx.x; c0 < (all + 63) / 64 * 64; c0 += P8_U * stride) {
        Raw8 r[P8_U];
        int64_t row[P8_U];
        int col[P8_U];
#pragma unroll
        for (int u = 0; u < P8_U; ++u) {
            const int64_t c = c0 + u * stride;
            // (32 bits are enough for the chunks of nearly all matrices, and divide much faster)
            if (all <= UINT32_MAX) row[u] = (uint32_t)c / (uint32_t)per;
            else row[u] = c / per;
            col[u] = (int)(c - row[u] * per) * 8;
            r[u] = Raw8{};
            if (c < all && col[u] < a.cols) r[u] = load_raw<X>((const T *)a.x + row[u] * a.ldx + col[u], a.cols - col[u]);
        }
        uint32_t most[P8_U], any = 0;
#pragma unroll
        for (int u = 0; u < P8_U; ++u) {
            uint32_t m[4];
            magnitudes<X, false>(r[u], m);
            most[u] = most_of(m), any = max2(any, most[u]);
        }
        auto put = [&](auto odd) {
            constexpr bool ODD = decltype(odd)::value;
#pragma unroll
            for (int u = 0; u < P8_U; ++u) {
                if (ODD) {
                    uint32_t m[4];
                    magnitudes<X, true>(r[u], m);
                    most[u] = most_of(m);
                }
                const int e = exp_of<X>(both(max16(most[u])) & 0xFFFFu), block = col[u] / E8_BLOCK;
                if (c0 + u * stride >= all) continue;
                *(uint2 *)(a.to.codes + row[u] * a.to.ld + col[u]) = codes8<X, ODD>(r[u], down(e));
                if (col[u] % E8_BLOCK == 0) {
                    a.to.exps[row[u] * a.to.lde + block] = (uint8_t)(e + E8_BIAS);
                    if (block + 1 == per / 16) pad_exps(a.to, row[u], per / 16);
                }
            }
        };
        if (any_odd<X>(any)) put(std::true_type{});
        else put(std::false_type{});
    }
}

// Turned lines of a tile: unit u (8 bytes) of line l stands at place u ^ (l >> 3), so
// that the 16 lanes that write units of eight lines apart fall into different banks.
__device__ __forceinline__ uint2 *unit_at(uint8_t *lines, int line, int u) { return (uint2 *)(lines + line * E8_BLOCK + 8 * (u ^ (line >> 3))); }

// The turned lines of a tile to memory, 16 bytes a thread.
__device__ __forceinline__ void put_lines(uint8_t *lines, const Blocks &to, int tr, int tc, int32_t cols)
{
    __syncthreads();
    int line = (int)threadIdx.x >> 3;
    const int u = 2 * ((int)threadIdx.x & 7), left = cols - tc * E8_BLOCK;
    uint8_t *at = to.codes + ((int64_t)tc * E8_BLOCK + line) * to.ld + (int64_t)tr * E8_BLOCK + 8 * u;
#pragma unroll
    for (int i = 0; i < 4; ++i, line += P8_TPB / 8, at += P8_TPB / 8 * to.ld) {
        const uint2 lo = *unit_at(lines, line, u), hi = *unit_at(lines, line, u + 1);
        if (line < left) *(uint4 *)at = uint4{lo.x, lo.y, hi.x, hi.y};
    }
}

// Everything else.  A workgroup takes a tile of 128 x 128, a thread 8 rows of 8
// columns of it: the 16 lanes beside each other have a row's block, the 16 groups of
// them a column's.  Turned codes change places in LDS, so that both results are
// written in whole lines of 128 bytes.  Bound by the bytes (8192x4096 in bf16 across: 18.9
// us, 5.3 TB/s; 4096x11008 both ways and its sums 46 us, 3.9 TB/s: bands of tiles below
// each other, for longer runs of turned lines, do not change it).
template <class X, bool CODES> __global__ __launch_bounds__(P8_TPB) void k_pack8(Pack8Args a)
{
    typedef typename X::T T;
    __shared__ uint32_t most[4][E8_BLOCK / 2];
    __shared__ float sums[4][E8_BLOCK];
    __shared__ __attribute__((aligned(16))) uint8_t lines[E8_BLOCK * E8_BLOCK];
    const int lane = lane_id(), wave = wave_id(), rg = (int)threadIdx.x >> 4, cc = (int)threadIdx.x & 15;
    const int64_t tile = (int64_t)blockIdx.x + a.first;
    const int tr = (int)(tile / a.tiles_c), tc = (int)(tile % a.tiles_c);
    const int row0 = tr * E8_BLOCK + 8 * rg, col0 = tc * E8_BLOCK + 8 * cc, left = a.cols - col0;

    Raw8 v[8];
    const T *x = (const T *)a.x + (int64_t)row0 * a.ldx + col0;
    const uint8_t *from = a.from.codes + (int64_t)row0 * a.from.ld + col0, *from_e = a.from.exps + (int64_t)row0 * a.from.lde + tc;
#pragma unroll
    for (int i = 0; i < 8; ++i, x += a.ldx, from += a.from.ld, from_e += a.from.lde) {
        v[i] = Raw8{};
        if (row0 + i >= a.rows || left <= 0) continue;
        if constexpr (CODES) {
            float f[8];
            e8_values<X>(*(const uint2 *)from, (int)*from_e - E8_BIAS, f);
            typename X::V8 t;
#pragma unroll
            for (int j = 0; j < 8; ++j) t[j] = j < left ? (T)f[j] : (T)0.f;
            v[i] = __builtin_bit_cast(Raw8, t);
        } else v[i] = load_raw<X>(x, left);
    }
    // largest magnitudes: mr of the thread's rows, two to a word, mc of its columns
    uint32_t mr[4], mc[4];
    auto sizes = [&](auto odd) {
#pragma unroll
        for (int k = 0; k < 4; ++k) mr[k] = mc[k] = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t m[4];
            magnitudes<X, decltype(odd)::value>(v[i], m);
#pragma unroll
            for (int k = 0; k < 4; ++k) mc[k] = max2(mc[k], m[k]);
            const uint32_t r = both(most_of(m));
            mr[i >> 1] |= i & 1 ? r & 0xFFFF0000u : r & 0xFFFFu;
        }
    };
    sizes(std::false_type{});
    // (a way of its own, for a wave that has one)
    const bool odd = any_odd<X>(most_of(mc));
    if (odd) sizes(std::true_type{});
    if (a.tile || a.turned.codes || a.sums) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            mc[k] = max2(mc[k], (uint32_t)__shfl_xor((int)mc[k], 16, 64));
            mc[k] = max2(mc[k], (uint32_t)__shfl_xor((int)mc[k], 32, 64));
            if (lane < 16) most[wave][4 * cc + k] = mc[k];
        }
        if (a.sums)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float s = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) s += value16<X>(half_of(v[i], j));
                s += __shfl_xor(s, 16, 64);
                s += __shfl_xor(s, 32, 64);
                if (lane < 16) sums[wave][8 * cc + j] = s;
            }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 4; ++k)
            mc[k] = max2(max2(most[0][4 * cc + k], most[1][4 * cc + k]), max2(most[2][4 * cc + k], most[3][4 * cc + k]));
    }
    if (a.tile) {
        const uint32_t m = both(max16(max2(max2(mc[0], mc[1]), max2(mc[2], mc[3]))));
#pragma unroll
        for (int k = 0; k < 4; ++k) mr[k] = mc[k] = m;
    }
    if (a.sums && threadIdx.x < E8_BLOCK) {
        const int c = (int)threadIdx.x, col = tc * E8_BLOCK + c;
        if (col < a.cols) a.sums[tr * (int64_t)a.cols + col] = sums[0][c] + sums[1][c] + sums[2][c] + sums[3][c];
    }
    auto put = [&](auto odd_t) {
        uint8_t *to = a.to.codes + (int64_t)row0 * a.to.ld + col0, *exp = a.to.exps + (int64_t)(row0 >> a.to.shift) * a.to.lde + tc;
#pragma unroll
        for (int i = 0; i < 8; ++i, to += a.to.ld, exp += a.to.lde) {
            const int e = exp_of<X>(i & 1 ? mr[i >> 1] >> 16 : mr[i >> 1] & 0xFFFFu);
            if (row0 + i >= a.rows) continue;
            *(uint2 *)to = codes8<X, decltype(odd_t)::value>(v[i], down(e));
            if (cc == 0 && (!a.tile || (rg == 0 && i == 0))) {  // (of a tile one, the first)
                *exp = (uint8_t)(e + E8_BIAS);
                if (tc == a.tiles_c - 1) pad_exps(a.to, (int64_t)(row0 + i) >> a.to.shift, a.tiles_c);
            }
        }
    };
    auto turn = [&](auto odd_t) {
        constexpr bool ODD = decltype(odd_t)::value;
        uint8_t *exp = a.turned.exps + (int64_t)(col0 >> a.turned.shift) * a.turned.lde + tr;
#pragma unroll
        for (int j = 0; j < 8; ++j, exp += a.turned.lde) {
            const int e = exp_of<X>(j & 1 ? mc[j >> 1] >> 16 : mc[j >> 1] & 0xFFFFu);
            const float by = down(e);
            auto at = [&](int i) { return value16<X>(half_of(v[i], j)) * by; };
            *unit_at(lines, 8 * cc + j, rg) = uint2{codes4<ODD>(at(0), at(1), at(2), at(3)), codes4<ODD>(at(4), at(5), at(6), at(7))};
            if (rg == 0 && j < left && (!a.tile || (cc == 0 && j == 0))) {
                const int64_t blocks = e8_blocks(a.rows);
                *exp = (uint8_t)(e + E8_BIAS);
                if (tr == blocks - 1) pad_exps(a.turned, (int64_t)(col0 + j) >> a.turned.shift, blocks);
            }
        }
    };
    if (a.to.codes) {
#pragma unroll
        for (int k = 0; k < 4; ++k) mr[k] = max16(mr[k]);
        if (odd) put(std::true_type{});
        else put(std::false_type{});
    }
    if (a.turned.codes) {
        if (odd) turn(std::true_type{});
        else turn(std::false_type{});
        put_lines(lines, a.turned, tr, tc, a.cols);
    }
}

// A thread per chunk of eight columns.  Bound by the bytes (4096x8192 in bf16: 18.5 us,
// 5.4 TB/s).
template <class X>
__global__ __launch_bounds__(P8_TPB) void k_unpack8(Blocks b, int32_t rows, int32_t cols, int32_t per, typename X::T *y, int64_t ldy)
{
    const int64_t chunks = (int64_t)rows * per;
    for (int64_t c = (int64_t)blockIdx.x * P8_TPB + threadIdx.x; c < chunks; c += (int64_t)gridDim.x * P8_TPB) {
        const int64_t row = chunks <= UINT32_MAX ? (uint32_t)c / (uint32_t)per : c / per;
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

// Four rows of four bytes turned.
__device__ __forceinline__ void turn4(uint32_t (&w)[4])
{
    const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), b = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u);
    const uint32_t c = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u), d = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
    w[0] = __builtin_amdgcn_perm(c, a, 0x05040100u), w[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
    w[2] = __builtin_amdgcn_perm(d, b, 0x05040100u), w[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
}

// A tile of codes a workgroup, turned eight by eight in registers and then, line by
// line, in LDS; its exponent goes with it.  Bound by the bytes (11008x4096: 20.6 us, 4.4
// TB/s).
__global__ __launch_bounds__(P8_TPB) void k_turn8(Blocks b, int32_t rows, int32_t cols, int32_t tiles_c, int32_t first, Blocks to)
{
    __shared__ __attribute__((aligned(16))) uint8_t lines[E8_BLOCK * E8_BLOCK];
    const int64_t tile = (int64_t)blockIdx.x + first;
    const int tr = (int)(tile / tiles_c), tc = (int)(tile % tiles_c), rg = (int)threadIdx.x >> 4, cc = (int)threadIdx.x & 15;
    uint32_t w[2][2][4];  // [upper four rows][left four columns][row]
    const int row0 = tr * E8_BLOCK + 8 * rg;
    const uint8_t *from = b.codes + (int64_t)row0 * b.ld + (int64_t)tc * E8_BLOCK + 8 * cc;
#pragma unroll
    for (int i = 0; i < 8; ++i, from += b.ld) {
        uint2 v = {0, 0};
        if (row0 + i < rows) v = *(const uint2 *)from;
        w[i >> 2][0][i & 3] = v.x, w[i >> 2][1][i & 3] = v.y;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) turn4(w[i >> 1][i & 1]);
#pragma unroll
    for (int j = 0; j < 8; ++j) *unit_at(lines, 8 * cc + j, rg) = uint2{w[0][j >> 2][j & 3], w[1][j >> 2][j & 3]};
    put_lines(lines, to, tr, tc, cols);
    if (threadIdx.x == 0) {
        to.exps[(int64_t)tc * to.lde + tr] = b.exps[(int64_t)tr * b.lde + tc];
        const int64_t blocks = e8_blocks(rows);
        if (tr == blocks - 1) pad_exps(to, tc, blocks);
    }
}

constexpr int64_t MAX_TILES8 = 1 << 30;

hipError_t launch_pack8(bool bf16, Pack8Args a, int32_t cus, hipStream_t s)
{
    if (a.rows == 0 || a.cols == 0) return hipSuccess;
    const int64_t tiles = e8_blocks(a.rows) * e8_blocks(a.cols);
    if (tiles > MAX_TILES8) return hipErrorInvalidConfiguration;
    a.tiles_c = (int32_t)e8_blocks(a.cols);
    if (a.to.codes && !a.tile && !a.turned.codes && !a.sums && !a.from.codes) {
        const int64_t chunks = (int64_t)a.rows * a.tiles_c * 16;
        const dim3 grid((unsigned)std::min<int64_t>((chunks + P8_TPB - 1) / P8_TPB, 8 * (int64_t)cus));
        if (bf16) hipLaunchKernelGGL(k_pack8_rows<Bf16>, grid, dim3(P8_TPB), 0, s, a);
        else hipLaunchKernelGGL(k_pack8_rows<Fp16>, grid, dim3(P8_TPB), 0, s, a);
        return hipGetLastError();
    }
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
