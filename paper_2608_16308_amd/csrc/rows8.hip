// The product in 8-bit floating point for a few tokens: the weights are read once,
// straight into registers.
#include <algorithm>

#include "float8.hpp"

namespace dbs {

typedef int v8i_t __attribute__((ext_vector_type(8)));
typedef int v4i_t __attribute__((ext_vector_type(4)));

constexpr int R8_U = 8;               // blocks that a wave has on their way
constexpr int R8_WAVES = 8;
// Blocks of x that a workgroup packs itself, for each of its waves; above, a launch of
// its own does it once for all.  In here and with the launch, bf16: 4096->11008 (four
// waves), 1 token 11.2 and 15.1 us, 4 (32 a wave) 15.2 and 15.1, 8 21.1 and 16.8;
// 14336->4096 (eight), 2 tokens (28) 16.9 and 17.2; 28672->8192 (28) 49.4 and 54.9;
// 1024->4096 (one), 16 tokens (128) 19.5 and 14.1.
constexpr int64_t R8_PACK = 32;

struct Rows8Args {
    Mul8Args m;
    const void *x;
    int64_t ldx;
    int32_t first, blocks;
    int32_t ldl;  // bytes of a token in LDS: rows of 16 tokens start in different banks
};

// A workgroup takes 16 rows of p, its waves share the blocks along k; their sums are
// added in LDS, in their order.  x (RAW: 16-bit values) is brought into blocks in LDS
// while the first weights are on their way: a launch of its own would take as long as
// half of the product of one token.  Bound by the bytes of the weights (1 token,
// 4096->11008 in bf16: 11.2 us, 4.0 TB/s with the launch; 28672->8192 4.8 TB/s).
template <class X, bool RAW> __global__ __launch_bounds__(64 * R8_WAVES) void k_rows8(Rows8Args a)
{
    typedef typename X::T T;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const Mul8Args &m = a.m;
    const int lane = lane_id(), wave = wave_id(), waves = (int)blockDim.x / 64, r = lane & 15, g = lane >> 4;
    const int p0 = ((int)blockIdx.x + a.first) * 16, t = m.qn;
    const int b0 = (int)((int64_t)a.blocks * wave / waves), b1 = (int)((int64_t)a.blocks * (wave + 1) / waves);
    const uint8_t *w = m.p.codes + min(p0 + r, m.pn - 1) * m.p.ld + 16 * g;
    const uint8_t *pe = m.p.exps + (int64_t)(p0 >> m.p.shift) * m.p.lde;
    const int token = min(r, t - 1);
    const uint8_t *q = m.q.codes + token * m.q.ld + 16 * g, *qe = m.q.exps + token * m.q.lde;
    uint8_t *xs = lds, *xe = lds + (int64_t)t * a.ldl;

    v4i_t lo[R8_U], hi[R8_U], xl[R8_U], xh[R8_U];
    int se[R8_U];
    auto fetch = [&](int b) {
#pragma unroll
        for (int u = 0; u < R8_U; ++u)
            if (b + u < b1) {
                const int64_t at = (int64_t)(b + u) * E8_BLOCK;
                lo[u] = *(const v4i_t *)(w + at), hi[u] = *(const v4i_t *)(w + at + 64);
                if constexpr (!RAW) xl[u] = *(const v4i_t *)(q + at), xh[u] = *(const v4i_t *)(q + at + 64), se[u] = qe[b + u];
            }
    };
    fetch(b0);
    if constexpr (RAW) {
        // 16 lanes a block
        for (int i = (int)threadIdx.x >> 4; i < (t * a.blocks + 3) / 4 * 4; i += (int)blockDim.x >> 4) {
            const int row = i / a.blocks, b = i - row * a.blocks, col = b * E8_BLOCK + 8 * r;
            Raw8 v{};
            if (row < t && col < m.kn) v = load_raw<X>((const T *)a.x + row * a.ldx + col, m.kn - col);
            uint32_t mag[4];
            magnitudes<X, false>(v, mag);
            const bool odd = any_odd<X>(most_of(mag));
            if (odd) magnitudes<X, true>(v, mag);
            const int e = exp_of<X>(both(max16(most_of(mag))) & 0xFFFFu);
            if (row >= t) continue;
            *(uint2 *)(xs + row * a.ldl + col) = odd ? codes8<X, true>(v, down(e)) : codes8<X, false>(v, down(e));
            if (r == 0) xe[row * a.blocks + b] = (uint8_t)(e + E8_BIAS);
        }
        __syncthreads();
    }
    f4_t acc = {0.f, 0.f, 0.f, 0.f};
    for (int b = b0; b < b1; b += R8_U) {
#pragma unroll
        for (int u = 0; u < R8_U; ++u)
            if (b + u < b1) {
                if constexpr (RAW) {
                    const uint8_t *x = xs + token * a.ldl + (b + u) * E8_BLOCK + 16 * g;
                    xl[u] = *(const v4i_t *)x, xh[u] = *(const v4i_t *)(x + 64), se[u] = xe[token * a.blocks + b + u];
                }
                acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(__builtin_shufflevector(lo[u], hi[u], 0, 1, 2, 3, 4, 5, 6, 7),
                                                                       __builtin_shufflevector(xl[u], xh[u], 0, 1, 2, 3, 4, 5, 6, 7), acc, 0, 0, 0,
                                                                       (int)pe[b + u], 0, se[u]);
            }
        fetch(b + R8_U);
    }
    // lane (g, r) holds rows 4 g .. + 3 of p for token r
    __syncthreads();
    f4_t *sums = (f4_t *)lds;
    sums[wave * 64 + lane] = acc;
    __syncthreads();
    for (int c = (int)threadIdx.x; c < 256; c += (int)blockDim.x) {
        const int of = c >> 4, row = c & 15, col = p0 + row;
        if (of >= t || col >= m.pn) continue;
        const float *s = (const float *)lds + ((row >> 2) * 16 + of) * 4 + (row & 3);
        float v = s[0];
        for (int i = 1; i < waves; ++i) v += s[i * 256];
        if (m.bias) v += (float)((const T *)m.bias)[col];
        if (m.res) v += (float)((const T *)m.res)[of * m.ldr + col];
        ((T *)m.y)[of * m.ldy + col] = (T)v;
    }
}

static int64_t token_bytes(int64_t blocks) { return blocks * E8_BLOCK + 16; }

static int64_t rows8_waves(int64_t blocks) { return std::max<int64_t>(1, std::min<int64_t>(R8_WAVES, (blocks + R8_U - 1) / R8_U)); }
bool rows8_pack(int64_t tokens, int64_t cols)
{
    const int64_t blocks = e8_blocks(cols);
    return tokens <= ROWS8_TOKENS && tokens * blocks <= R8_PACK * rows8_waves(blocks);
}

template <class X> static hipError_t rows8_t(Rows8Args a, hipStream_t s)
{
    const int64_t groups = ((int64_t)a.m.pn + 15) / 16;
    const int waves = (int)rows8_waves(a.blocks);
    const int64_t x = a.x ? a.m.qn * ((int64_t)a.ldl + a.blocks) : 0;
    const unsigned lds = (unsigned)std::max<int64_t>(x, waves * 1024);
    return launch_parts(groups, 64 * waves, [&](int32_t first, dim3 grid) {
        a.first = first;
        if (a.x) hipLaunchKernelGGL((k_rows8<X, true>), grid, dim3((unsigned)(64 * waves)), lds, s, a);
        else hipLaunchKernelGGL((k_rows8<X, false>), grid, dim3((unsigned)(64 * waves)), lds, s, a);
    });
}

hipError_t launch_rows8(const LayerWork &w, bool bf16, const Mul8Args &m, const void *x, int64_t ldx, hipStream_t s)
{
    if (m.pn == 0 || m.qn == 0) return hipSuccess;
    Rows8Args a{m, x, ldx, 0, (int32_t)e8_blocks(m.kn), (int32_t)token_bytes(e8_blocks(m.kn))};
    return bf16 ? rows8_t<Bf16>(a, s) : rows8_t<Fp16>(a, s);
}

}  // namespace dbs
