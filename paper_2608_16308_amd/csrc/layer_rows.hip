// The forward products for a few tokens: the weights are read once, straight
// into registers, by workgroups that each take 16 rows of them.
#include <algorithm>

#include "device_common.hpp"
#include "layer.hpp"

namespace dbs {

template <class X> struct __attribute__((packed, aligned(2))) Eight {
    typename X::V8 v;
};
template <class X> __device__ __forceinline__ typename X::V8 load_eight(const typename X::T *p)
{
    return ((const Eight<X> *)p)->v;
}
// Eight elements, of which the first `left` exist.
template <class X> __device__ __forceinline__ typename X::V8 load_some(const typename X::T *p, int left)
{
    if (left >= 8) return load_eight<X>(p);
    typename X::V8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < left ? p[i] : (typename X::T)0.f;
    return v;
}

constexpr int RW_U = 8;               // products of 32 k in flight
constexpr int RW_K = 32 * RW_U;       // k of a wave's turn
constexpr int RW_MAX_WAVES = 16;

// A wave multiplies 16 rows of w (RG times 16; gated: of both matrices) with
// 16 TT tokens over its turns of RW_K elements; the waves' sums are added in
// LDS, in their order.  Rows past the last are read as the last one, and not
// written.
template <class X, bool GATED, int RG, int TT>
__global__ __launch_bounds__(64 * RW_MAX_WAVES) void k_rows_dense(GemmArgs a)
{
    typedef typename X::T T;
    typedef typename X::V8 V8;
    constexpr int NG = RG * (GATED ? 2 : 1), COLS = 16 * RG;
    extern __shared__ float sums[];  // [waves][NG][TT][4][64], then the totals [NG][16 TT][16]
    const int lane = lane_id(), wave = wave_id(), waves = (int)blockDim.x / 64, r = lane & 15, g = lane >> 4;
    const int p0 = (int)blockIdx.x * COLS;
    const T *w[NG], *x[TT];
#pragma unroll
    for (int n = 0; n < NG; ++n) {
        const int mat = GATED ? n / RG : 0;
        w[n] = (const T *)a.p[mat] + (int64_t)min(p0 + 16 * (n % RG) + r, a.pn - 1) * a.ldp[mat] + 8 * g;
    }
#pragma unroll
    for (int t = 0; t < TT; ++t) x[t] = (const T *)a.q[0] + (int64_t)min(16 * t + r, a.qn - 1) * a.ldq[0] + 8 * g;
    f4_t acc[NG][TT];
#pragma unroll
    for (int n = 0; n < NG; ++n)
#pragma unroll
        for (int t = 0; t < TT; ++t) acc[n][t] = f4_t{0.f, 0.f, 0.f, 0.f};

    int k = wave * RW_K;
    for (; k + RW_K <= a.kn; k += waves * RW_K) {
        V8 vw[NG][RW_U], vx[TT][RW_U];
#pragma unroll
        for (int n = 0; n < NG; ++n)
#pragma unroll
            for (int u = 0; u < RW_U; ++u) vw[n][u] = load_eight<X>(w[n] + k + 32 * u);
#pragma unroll
        for (int t = 0; t < TT; ++t)
#pragma unroll
            for (int u = 0; u < RW_U; ++u) vx[t][u] = load_eight<X>(x[t] + k + 32 * u);
#pragma unroll
        for (int u = 0; u < RW_U; ++u)
#pragma unroll
            for (int n = 0; n < NG; ++n)
#pragma unroll
                for (int t = 0; t < TT; ++t) acc[n][t] = X::mma(vw[n][u], vx[t][u], acc[n][t]);
    }
    if (k < a.kn)  // the last turn, ragged
        for (int u = 0; u < RW_U && k + 32 * u < a.kn; ++u) {
            const int left = a.kn - (k + 32 * u + 8 * g);
            V8 vx[TT];
#pragma unroll
            for (int t = 0; t < TT; ++t) vx[t] = load_some<X>(x[t] + k + 32 * u, left);
#pragma unroll
            for (int n = 0; n < NG; ++n) {
                const V8 vw = load_some<X>(w[n] + k + 32 * u, left);
#pragma unroll
                for (int t = 0; t < TT; ++t) acc[n][t] = X::mma(vw, vx[t], acc[n][t]);
            }
        }

    // lane (g, r) holds rows 4 g .. + 3 of w for token r
#pragma unroll
    for (int n = 0; n < NG; ++n)
#pragma unroll
        for (int t = 0; t < TT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) sums[(((wave * NG + n) * TT + t) * 4 + i) * 64 + lane] = acc[n][t][i];
    __syncthreads();
    float *total = sums + waves * NG * TT * 256;
    for (int c = (int)threadIdx.x; c < NG * TT * 256; c += (int)blockDim.x) {
        float s = sums[c];
        for (int v = 1; v < waves; ++v) s += sums[v * NG * TT * 256 + c];
        // c = ((n TT + t) 4 + i) 64 + 16 g + r: column 4 g + i of token 16 t + r
        const int l = c & 63, i = (c >> 6) & 3, nt = c >> 8;
        total[((nt / TT) * TT + nt % TT) * 256 + (l & 15) * 16 + 4 * (l >> 4) + i] = s;
    }
    __syncthreads();
    // a thread per token and column, a row of COLS columns in neighbouring lanes
    const int64_t ngroup = (a.pn + CK_GROUP - 1) / CK_GROUP;
    for (int c = (int)threadIdx.x; c < 16 * TT * COLS; c += (int)blockDim.x) {
        const int token = c / COLS, cc = c % COLS, col = p0 + cc;
        const bool in = token < a.qn && col < a.pn;
        auto value = [&](int mat) { return total[((mat * RG + cc / 16) * TT + token / 16) * 256 + (token & 15) * 16 + (cc & 15)]; };
        auto save = [&](const SaveTo &to, float v) {
            const T q = (T)v;
            if (to.full) {
                if (in) ((T *)to.full)[(int64_t)token * to.ld + col] = q;
            } else if (RG == 2) {
                float big = in ? ck_mag((float)q) : 0.f;
#pragma unroll
                for (int o = 1; o < CK_GROUP; o <<= 1) big = fmaxf(big, __shfl_xor(big, o, 64));
                if (!in) return;
                const int e = ck_exp<X>(big);
                to.codes[(int64_t)token * a.pn + col] = (int8_t)ck_code((float)q, e);
                if (cc == 0) to.exps[token * ngroup + col / CK_GROUP] = (uint8_t)(e + CK_BIAS);
            }
        };
        float v[1] = {value(0)};
        if (GATED) {
            const float up = value(1);
            if (a.save[0].full || a.save[0].codes) {
                save(a.save[0], v[0]);
                save(a.save[1], up);
            }
            act_values(a.act, v);
            v[0] *= up;
        } else {
            if (a.bias && in) v[0] += (float)((const T *)a.bias)[col];
            if (a.save[0].full || a.save[0].codes) save(a.save[0], v[0]);
            act_values(a.act, v);
            if (a.res && in) v[0] += (float)((const T *)a.res)[(int64_t)token * a.ldr + col];
        }
        if (in) ((T *)a.y[0])[(int64_t)token * a.ldy[0] + col] = (T)v[0];
    }
}

// Waves of a workgroup: a turn each at least, and no more than fill the device
// (each wave has RW_U loads of 1 KB in flight).
static int waves_of(const LayerWork &w, int64_t groups, int64_t kn)
{
    const int64_t turns = (kn + RW_K - 1) / RW_K, want = (16 * (int64_t)w.cus + groups - 1) / groups;
    int64_t n = std::max<int64_t>(1, std::min<int64_t>({turns, std::max<int64_t>(want, 4), RW_MAX_WAVES}));
    return (int)n;
}

template <class X, bool GATED, int RG, int TT> static hipError_t rows_t(const LayerWork &w, const GemmArgs &a, hipStream_t s)
{
    constexpr int NG = RG * (GATED ? 2 : 1);
    const int64_t groups = ((int64_t)a.pn + 16 * RG - 1) / (16 * RG);
    const int waves = waves_of(w, groups, a.kn);
    hipLaunchKernelGGL((k_rows_dense<X, GATED, RG, TT>), dim3((unsigned)groups), dim3((unsigned)(64 * waves)),
                       (size_t)(waves + 1) * NG * TT * 1024, s, a);
    return hipGetLastError();
}

template <class X, bool GATED> static hipError_t rows_g(const LayerWork &w, const GemmArgs &a, hipStream_t s)
{
    // a group of a checkpoint is 32 columns
    if (a.save[0].codes) return a.qn <= 16 ? rows_t<X, GATED, 2, 1>(w, a, s) : rows_t<X, GATED, 2, 2>(w, a, s);
    return a.qn <= 16 ? rows_t<X, GATED, 1, 1>(w, a, s) : rows_t<X, GATED, 1, 2>(w, a, s);
}

hipError_t launch_rows(const LayerWork &w, bool bf16, bool gated, const GemmArgs &a, hipStream_t s)
{
    if (a.qn == 0 || a.pn == 0) return hipSuccess;
    if (gated) return bf16 ? rows_g<Bf16, true>(w, a, s) : rows_g<Fp16, true>(w, a, s);
    return bf16 ? rows_g<Bf16, false>(w, a, s) : rows_g<Fp16, false>(w, a, s);
}

}  // namespace dbs
