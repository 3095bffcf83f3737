// Shared parts of the dense layer operators: element types, activations, the
// 8-bit checkpoint code, kernel arguments and launchers.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/dbspmspv.h"

namespace dbs {

typedef float f4_t __attribute__((ext_vector_type(4)));

// The two element types.  V8 is a 16-byte chunk of them, and mma() one
// 16x16x32 step on the matrix cores: lane l gives row l % 16 of a and column
// l % 16 of b, elements 8 (l / 16) .. + 7 of the sum, and holds rows
// 4 (l / 16) .. + 3 of column l % 16 of the 32-bit result.
struct Bf16 {
    typedef __bf16 T;
    typedef __bf16 V8 __attribute__((ext_vector_type(8)));
    typedef __bf16 V4 __attribute__((ext_vector_type(4)));
    static constexpr float MAX = 3.38953138925153547590470800371487867e38f;
    static constexpr int LEAST_EXP = -127;
    __device__ static __forceinline__ f4_t mma(V8 a, V8 b, f4_t c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
};
struct Fp16 {
    typedef _Float16 T;
    typedef _Float16 V8 __attribute__((ext_vector_type(8)));
    typedef _Float16 V4 __attribute__((ext_vector_type(4)));
    static constexpr float MAX = 65504.f;
    static constexpr int LEAST_EXP = -24;
    __device__ static __forceinline__ f4_t mma(V8 a, V8 b, f4_t c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    }
};

// Eight elements at any alignment.
template <class X> struct __attribute__((packed, aligned(2))) Eight {
    typename X::V8 v;
};
template <class X> __device__ __forceinline__ typename X::V8 load_eight(const typename X::T *p)
{
    return ((const Eight<X> *)p)->v;
}
// Elements k .. k + 7 of a row of n >= 8, zeros past its end: what stands at
// its last eight, moved down.
template <class X> __device__ __forceinline__ typename X::V8 load_end(const typename X::T *row, int k, int n)
{
    const int at = min(k, n - 8), by = k - at;
    struct Two {
        uint64_t lo, hi;
    } v = __builtin_bit_cast(Two, load_eight<X>(row + at));
    if (by >= 4) v.lo = v.hi, v.hi = 0;
    const int bits = 16 * (by & 3);
    v.lo = v.lo >> bits | (v.hi << 1) << (63 - bits);
    v.hi >>= bits;
    if (by >= 8) v.lo = v.hi = 0;
    return __builtin_bit_cast(typename X::V8, v);
}

// ---------------------------------------------------------------------------
// activations
// ---------------------------------------------------------------------------
// act(z).  SiLU is z times a logistic of z, and so is the tanh form of GELU, of
// a z + b z^3 (1 + tanh(q) = 2 logistic(2 q)), which also keeps the relative
// precision of the small values left of zero; GELU itself takes the complement
// of erf, 1 + erf(x) = erfc(-x): the sum would cancel there (4% off at -5).
struct Act {
    int32_t kind;
    static Act of(dbs_act k) { return Act{(int32_t)k}; }
};
constexpr float GELU_A = 1.5957691216057308f, GELU_B = GELU_A * 0.044715f;  // a = 2 sqrt(2 / pi)
__device__ __forceinline__ float logistic(float q) { return __builtin_amdgcn_rcpf(1.f + __expf(-q)); }

// v = act(v) for N values
template <int N> __device__ __forceinline__ void act_values(Act f, float (&v)[N])
{
    if (f.kind == DBS_ACT_NONE) return;
    if (f.kind == DBS_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = v[i] < 0.f ? 0.f : v[i];
    } else if (f.kind == DBS_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = 0.5f * v[i] * erfcf(v[i] * -0.70710678118654752f);
    } else if (f.kind == DBS_ACT_SILU) {  // (not the form below with b = 0: an infinite square times zero is NaN)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = v[i] * logistic(v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = v[i] * logistic(v[i] * (GELU_A + GELU_B * v[i] * v[i]));
    }
}
// Value and slope of z logistic(q), `g` the slope of q.  Where the logistic is 0
// or 1 the second term of the slope is 0, also where g has overflowed.
__device__ __forceinline__ void logistic_slope(float z, float q, float g, float &value, float &slope)
{
    const float s = logistic(q), d = s * (1.f - s);
    value = z * s;
    slope = s + (d == 0.f ? 0.f : z * d * g);
}
// act(z) and act'(z) of N values.
template <int N> __device__ __forceinline__ void act_slopes(Act f, const float (&z)[N], float (&value)[N], float (&slope)[N])
{
    if (f.kind == DBS_ACT_NONE) {
#pragma unroll
        for (int i = 0; i < N; ++i) value[i] = z[i], slope[i] = 1.f;
    } else if (f.kind == DBS_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) value[i] = z[i] < 0.f ? 0.f : z[i], slope[i] = z[i] > 0.f ? 1.f : 0.f;
    } else if (f.kind == DBS_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float c = 0.5f * erfcf(z[i] * -0.70710678118654752f);
            value[i] = z[i] * c;
            slope[i] = c + z[i] * __expf(-0.5f * z[i] * z[i]) * 0.39894228040143268f;
        }
    } else if (f.kind == DBS_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < N; ++i) logistic_slope(z[i], z[i], 1.f, value[i], slope[i]);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float zz = z[i] * z[i];
            logistic_slope(z[i], z[i] * (GELU_A + GELU_B * zz), GELU_A + 3.f * GELU_B * zz, value[i], slope[i]);
        }
    }
}

// ---------------------------------------------------------------------------
// 8-bit checkpoints
// ---------------------------------------------------------------------------
// A group of CK_GROUP columns of a row shares the exponent e, the least with
// a <= 127 * 2^e for the largest finite magnitude a; a value is the whole
// number nearest to v * 2^-e (ties to even), and -128 stands for a value that
// is not finite.  A scale that is a power of two costs up to one of the seven
// bits against a / 127, but every code * 2^e is a number of the 16-bit type,
// so what the backward pass multiplies is what the checkpoint holds, with no
// second rounding.
constexpr int CK_GROUP = 32;
constexpr int CK_BIAS = 127;

// The finite magnitude of v, 0 if it is not finite.
__device__ __forceinline__ float ck_mag(float v)
{
    const float a = __builtin_fabsf(v);
    return a <= 3.402823466e38f ? a : 0.f;
}
// e of a group with largest magnitude a.
template <class X> __device__ __forceinline__ int ck_exp(float a)
{
    const int k = __builtin_amdgcn_frexp_expf(a);         // a = m 2^k, m in [1/2, 1)
    const float m = __builtin_amdgcn_frexp_mantf(a);
    const int e = m <= 127.f / 128.f ? k - 7 : k - 6;
    return a == 0.f || e < X::LEAST_EXP ? X::LEAST_EXP : e;
}
__device__ __forceinline__ int ck_code(float v, int e)
{
    const float c = __builtin_rintf(__builtin_amdgcn_ldexpf(v, -e));
    return __builtin_fabsf(v) <= 3.402823466e38f ? (int)c : -128;
}
// The values of eight codes of a group.  The largest magnitudes reach 64 * 2^e =
// 2^(e + 6) beyond the type's largest number: such values come back as that
// number.
struct __attribute__((packed, aligned(1))) Codes8 {
    uint32_t w[2];
};
template <class X> __device__ __forceinline__ void ck_values(Codes8 c, int e, float (&v)[8])
{
    const float scale = __builtin_amdgcn_ldexpf(1.f, e);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t w = c.w[h] ^ 0x80808080u;  // code + 128
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float code = (float)((w >> (8 * i)) & 255u) - 128.f;
            v[4 * h + i] = __builtin_amdgcn_fmed3f(code * scale, -X::MAX, X::MAX);
        }
        if ((w - 0x01010101u) & ~w & 0x80808080u)  // a code of -128
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (((w >> (8 * i)) & 255u) == 0u) v[4 * h + i] = __builtin_nanf("");
    }
}

// ---------------------------------------------------------------------------
// kernel arguments
// ---------------------------------------------------------------------------
// Where an epilogue keeps 16-bit roundings of its sums: as they are, or as a
// checkpoint (rows of `cols` codes, contiguous).
struct SaveTo {
    void *full;
    int64_t ld;
    int8_t *codes;
    uint8_t *exps;
};
// What a backward pass reads: 16-bit values, or a checkpoint.
struct HeldIn {
    const void *full;
    int64_t ld;
    const int8_t *codes;
    const uint8_t *exps;
};

enum GemmKind { G_LINEAR, G_GATED, G_DX, G_DW };

// One product: Y[q][p] = sum over k of Q[q][k] P[p][k], Y row-major with p
// along its rows.
//   G_LINEAR  P = w, Q = x; epilogue act(. + bias) + residual
//   G_GATED   P = the rows of w_gate and w_up in turns, Q = x; act(gate) * up
//   G_DX      Q = dz, P[p][k] = w[k][p]; the sum runs over `segs` pairs
//   G_DW      Q[q][k] = dz[k][q], P[p][k] = x[k][p], k a token; `batch` pairs
struct GemmArgs {
    const void *p[2], *q[2];
    int64_t ldp[2], ldq[2];
    int32_t pn, qn, kn;      // sizes; pn of one matrix, kn of one pair
    int32_t segs, batch;
    void *y[2];
    int64_t ldy[2];
    const void *bias, *res;
    int64_t ldr;
    Act act;
    SaveTo save[2];
    int32_t p_padded, q_padded;  // rows of P, Q go on to a whole 16 bytes (Q of G_DX: with zeros)
    // filled by the launcher
    int32_t first;           // number of the launch's first workgroup
    int32_t chunks;          // P and Q are made of whole 16-byte chunks
    int32_t tp, tq;          // tiles along p and q
    int32_t full, splits;    // tiles taken whole; parts of each of the others along k
    const float *scale;      // G_DX, G_DW: what the sums are multiplied by (NULL: 1)
    float *part;             // the parts' sums
    const void *zeros;       // 16 bytes of zeros
};

// Launches `n` workgroups in parts of fewer than 2^32 threads, which is what the
// runtime takes: launch(first, number).
template <class F> static hipError_t launch_parts(int64_t n, int threads, F &&launch)
{
    const int64_t most = (UINT32_MAX / threads) & ~(int64_t)7;  // (each XCD as in one launch)
    for (int64_t first = 0; first < n; first += most) {
        launch((int32_t)first, dim3((unsigned)(n - first < most ? n - first : most)));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// Workspace of a layer context.
struct LayerWork {
    float *part;
    size_t part_bytes;
    const void *zeros;
    int32_t cus;
};

hipError_t launch_gemm(const LayerWork &w, bool bf16, GemmKind kind, GemmArgs a, hipStream_t s);
// Whether an operand is made of whole 16-byte chunks (`contiguous` of its
// elements in a row), as loads straight into LDS need it, near enough to each
// other for 32-bit offsets within a tile.
bool whole_chunks(const void *p, int64_t ld, int64_t contiguous);
// A copy of an operand in rows of ldd elements, zeros behind the last column.
hipError_t launch_align(const void *src, int64_t ld, int32_t rows, int32_t cols, void *dst, int64_t ldd, int32_t cus,
                        hipStream_t s);

// G_LINEAR and G_GATED for few tokens; whether these kernels take a call: up to
// ROWS_TOKENS tokens, rows of at least a load, 16 of them within 32-bit offsets.
constexpr int ROWS_TOKENS = 16;
bool rows_take(bool gated, const GemmArgs &a);
hipError_t launch_rows(const LayerWork &w, bool bf16, bool gated, const GemmArgs &a, hipStream_t s);

// Activation gradients: dz = dy * act'(pre) or, gated, dz = dy * up * act'(gate)
// and du = dy * act(gate), rounded to the element type, rows of `ldz` elements
// with zeros behind the last column; sums of the columns of the unrounded dz.
//
// Why 16 bits: dz and du are operands of the matrix cores.  That costs a rounding
// of u of each of them (in bf16 the gradients are then 2.3e-3 from 64 bits, where
// the final rounding alone is 1.7e-3; in fp16 2.9e-4 and 2.1e-4); two 16-bit parts
// for each would double the products.  In fp16 such a product of 16-bit numbers may
// leave the type's range where the gradients do not, so there all dz and du of a
// call are held times a power of two 2^-s, and the sums over them are multiplied by
// 2^s in 32 bits: see slope_exp.
struct SlopeArgs {
    const void *dy;
    int64_t lddy;
    HeldIn pre, up;
    int32_t rows, cols;
    Act act;
    void *dz, *du;      // dz NULL: only the sums
    int64_t ldz;
    float *sums;        // NULL, or row_blocks x cols
    void *db;
    int32_t row_blocks; // workgroups along the rows
    float *most;        // NULL, or for each workgroup its largest |dz|, |du|, and then 2^s
};
// s for the largest finite magnitude m of dz and du: 0 while they keep to the
// range (from 2^-8 on, what is lost below the least fp16 number is under 2^-17 of
// m), else m 2^-s is in [2^14, 2^15); s >= -60 keeps 2^s a normal number.
__device__ __forceinline__ int slope_exp(float m)
{
    if (m == 0.f || (m >= 0.00390625f && m <= Fp16::MAX)) return 0;
    return max((int)__builtin_amdgcn_frexp_expf(m) - 15, -60);
}
int32_t slope_row_blocks(int32_t rows, int32_t cols, int32_t cus);
// Workgroups of a call (the elements of `most` before 2^s).
int64_t slope_blocks(int32_t rows, int32_t cols, int32_t cus);
hipError_t launch_slope(bool bf16, bool gated, const SlopeArgs &a, hipStream_t s);

hipError_t launch_pack(bool bf16, const void *x, int64_t ldx, int32_t rows, int32_t cols, int8_t *codes, uint8_t *exps,
                       int32_t cus, hipStream_t s);
hipError_t launch_unpack(bool bf16, const int8_t *codes, const uint8_t *exps, int32_t rows, int32_t cols, void *y,
                         int64_t ldy, int32_t cus, hipStream_t s);

}  // namespace dbs
