// Blocks of 8-bit floating point: their codes, scales and places in memory.
#pragma once
#include "device_common.hpp"
#include "layer.hpp"

namespace dbs {

// A block of E8_BLOCK columns (of a row, or of E8_BLOCK rows) shares the
// exponent e, the least with a <= 448 * 2^e for its largest finite magnitude a; a
// value is the e4m3 number nearest to v * 2^-e (ties to even), NaN if it is not
// finite.  448 is the largest e4m3 number.  A scale that is a power of two costs
// nothing here that a / 448 would keep: the codes are floating point themselves,
// so a value has its four bits wherever it lies in their range (of which up to
// one of 17 binades is given up), and the matrix cores apply such scales
// themselves.
constexpr int E8_BLOCK = 128;
constexpr int E8_BIAS = 127;
constexpr float E8_MAX = 448.f;

// e of a block with largest finite magnitude a.
__device__ __forceinline__ int e8_exp(float a)
{
    const int k = __builtin_amdgcn_frexp_expf(a);  // a = m 2^k, m in [1/2, 1); 448 = 7/8 2^9
    const int e = __builtin_amdgcn_frexp_mantf(a) <= 0.875f ? k - 9 : k - 8;
    return a == 0.f || e < -E8_BIAS ? -E8_BIAS : e;
}
// v * 2^-e as it is rounded; NaN if v is not finite.
__device__ __forceinline__ float e8_scaled(float v, int e)
{
    return __builtin_fabsf(v) <= 3.402823466e38f ? __builtin_amdgcn_ldexpf(v, -e) : __builtin_nanf("");
}
// The codes of eight values.
__device__ __forceinline__ uint2 e8_codes(const float (&v)[8], int e)
{
    int w[2] = {0, 0};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        w[h] = __builtin_amdgcn_cvt_pk_fp8_f32(e8_scaled(v[4 * h], e), e8_scaled(v[4 * h + 1], e), w[h], false);
        w[h] = __builtin_amdgcn_cvt_pk_fp8_f32(e8_scaled(v[4 * h + 2], e), e8_scaled(v[4 * h + 3], e), w[h], true);
    }
    return uint2{(uint32_t)w[0], (uint32_t)w[1]};
}
// The values of eight codes, limited to the finite numbers of the 16-bit type
// (the largest of a block may reach the next power of two beyond them).
template <class X> __device__ __forceinline__ void e8_values(uint2 c, int e, float (&v)[8])
{
    const int w[2] = {(int)c.x, (int)c.y};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        v[4 * h] = __builtin_amdgcn_cvt_f32_fp8(w[h], 0), v[4 * h + 1] = __builtin_amdgcn_cvt_f32_fp8(w[h], 1);
        v[4 * h + 2] = __builtin_amdgcn_cvt_f32_fp8(w[h], 2), v[4 * h + 3] = __builtin_amdgcn_cvt_f32_fp8(w[h], 3);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float s = __builtin_amdgcn_ldexpf(v[i], e);
        v[i] = s > X::MAX ? X::MAX : s < -X::MAX ? -X::MAX : s;  // (NaN stays)
    }
}

// Magnitudes are compared as the integers that their 16 bits are, two to a word.
typedef uint16_t h2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b)
{
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(h2_t, a), __builtin_bit_cast(h2_t, b)));
}
template <class X> struct Bits;  // of infinity
template <> struct Bits<Bf16> {
    static constexpr uint32_t INF = 0x7F80u;
};
template <> struct Bits<Fp16> {
    static constexpr uint32_t INF = 0x7C00u;
};
// The larger of a word's halves, in both.
__device__ __forceinline__ uint32_t both(uint32_t m) { return max2(m, m >> 16 | m << 16); }
// The largest of 16 neighbouring lanes, by halves.
__device__ __forceinline__ uint32_t max16(uint32_t m)
{
    m = max2(m, dpp_mov<dppc::ROW_ROR + 1>(0u, m));
    m = max2(m, dpp_mov<dppc::ROW_ROR + 2>(0u, m));
    m = max2(m, dpp_mov<dppc::ROW_ROR + 4>(0u, m));
    return max2(m, dpp_mov<dppc::ROW_ROR + 8>(0u, m));
}
template <class X> __device__ __forceinline__ float value16(uint32_t bits)
{
    return (float)__builtin_bit_cast(typename X::T, (uint16_t)bits);
}
// A block's exponent from the bits of its largest magnitude.
template <class X> __device__ __forceinline__ int exp_of(uint32_t bits) { return e8_exp(value16<X>(bits)); }
// 2^-e (a normal number: -127 <= e <= 120)
__device__ __forceinline__ float down(int e) { return __builtin_bit_cast(float, (uint32_t)(127 - e) << 23); }
// Four values as codes.  A value that is not finite becomes NaN (ODD: where one may be
// among them).
__device__ __forceinline__ float finite_or_nan(float v) { return __builtin_fabsf(v) <= 3.402823466e38f ? v : __builtin_nanf(""); }
template <bool ODD> __device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d)
{
    if (ODD) a = finite_or_nan(a), b = finite_or_nan(b), c = finite_or_nan(c), d = finite_or_nan(d);
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    return (uint32_t)w;
}
// Eight 16-bit numbers; the words of their magnitudes, not finite ones as zeros.
struct Raw8 {
    uint32_t w[4];
};
template <class X, bool ODD> __device__ __forceinline__ void magnitudes(const Raw8 &r, uint32_t (&m)[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m[i] = r.w[i] & 0x7FFF7FFFu;
        if (!ODD) continue;
        if ((m[i] & 0xFFFFu) >= Bits<X>::INF) m[i] &= 0xFFFF0000u;
        if (m[i] >> 16 >= Bits<X>::INF) m[i] &= 0xFFFFu;
    }
}
__device__ __forceinline__ uint32_t most_of(const uint32_t (&m)[4]) { return max2(max2(m[0], m[1]), max2(m[2], m[3])); }
// Whether a half of the word, a largest magnitude, is not finite, in any lane.
template <class X> __device__ __forceinline__ bool any_odd(uint32_t m) { return ballot((both(m) & 0xFFFFu) >= Bits<X>::INF) != 0; }
template <class X> __device__ __forceinline__ Raw8 load_raw(const typename X::T *p, int left)
{
    if (left >= 8) return __builtin_bit_cast(Raw8, load_eight<X>(p));
    typename X::V8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < left ? p[i] : (typename X::T)0.f;
    return __builtin_bit_cast(Raw8, v);
}
__device__ __forceinline__ uint32_t half_of(const Raw8 &r, int i) { return i & 1 ? r.w[i >> 1] >> 16 : r.w[i >> 1] & 0xFFFFu; }
template <class X, bool ODD> __device__ __forceinline__ uint2 codes8(const Raw8 &r, float by)
{
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
        w[h] = codes4<ODD>(value16<X>(half_of(r, 4 * h)) * by, value16<X>(half_of(r, 4 * h + 1)) * by, value16<X>(half_of(r, 4 * h + 2)) * by,
                           value16<X>(half_of(r, 4 * h + 3)) * by);
    return uint2{w[0], w[1]};
}
// Codes of a matrix: rows of whole blocks, zeros behind the last column.
// Exponents + 127: for each row (or E8_BLOCK rows) one byte for each block, rows
// of whole fours, 127 behind the last.
__host__ __device__ __forceinline__ int64_t e8_blocks(int64_t cols) { return (cols + E8_BLOCK - 1) / E8_BLOCK; }
__host__ __device__ __forceinline__ int64_t e8_ld(int64_t cols) { return e8_blocks(cols) * E8_BLOCK; }
__host__ __device__ __forceinline__ int64_t e8_ldexp(int64_t cols) { return (e8_blocks(cols) + 3) / 4 * 4; }

// A matrix of `rows` rows in blocks.
struct Blocks {
    uint8_t *codes, *exps;
    int64_t ld, lde;
    int32_t shift;  // exponents of row r stand in row r >> shift
};

// x (16-bit values, or row blocks) into blocks: of x, of its transpose, or both
// in one pass; the sums of its columns over each E8_BLOCK rows.
struct Pack8Args {
    const void *x;
    int64_t ldx;
    Blocks from;    // x as row blocks (codes not NULL)
    int32_t rows, cols;
    int32_t tile;   // one exponent for each tile
    Blocks to, turned;  // codes NULL: not wanted
    float *sums;    // NULL, or [ceil(rows / E8_BLOCK)][cols]
    int32_t tiles_c, first;  // filled by the launcher
};
hipError_t launch_pack8(bool bf16, Pack8Args a, int32_t cus, hipStream_t s);
hipError_t launch_unpack8(bool bf16, const Blocks &b, int32_t rows, int32_t cols, void *y, int64_t ldy, int32_t cus, hipStream_t s);
// The transpose of a matrix in tile blocks.
hipError_t launch_turn8(const Blocks &b, int32_t rows, int32_t cols, const Blocks &to, hipStream_t s);

// y = q p^T + bias + res: p [pn, kn], q [qn, kn] in blocks along k.
struct Mul8Args {
    Blocks p, q;
    int32_t pn, qn, kn;
    const void *bias, *res;
    int64_t ldr;
    void *y;
    int64_t ldy;
};
// The same for up to ROWS8_TOKENS rows of q, given in blocks or (x not NULL) as 16-bit
// values, which the kernel brings into blocks itself where they fit its LDS.
constexpr int ROWS8_TOKENS = 16;
bool rows8_pack(int64_t tokens, int64_t cols);
hipError_t launch_rows8(const LayerWork &w, bool bf16, const Mul8Args &m, const void *x, int64_t ldx, hipStream_t s);
hipError_t launch_mul8(const LayerWork &w, bool bf16, const Mul8Args &m, hipStream_t s);

}  // namespace dbs
