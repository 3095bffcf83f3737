// Norms, joins and dropout: arguments, launchers and what their kernels share.
#pragma once
#include "device_common.hpp"
#include "layer.hpp"

namespace dbs {

// ---------------------------------------------------------------------------
// dropout
// ---------------------------------------------------------------------------
// An element is dropped where its 16 random bits are below `threshold`, and
// multiplied by `scale` elsewhere.  The bits are a function of its place and of
// (seed, offset) alone, so the backward pass makes them again and no mask is
// stored.
struct Drop {
    uint32_t threshold;  // 0: nothing is dropped
    float scale;
    uint64_t seed, offset;
    const uint64_t *rng;  // NULL, or seed and offset in device memory
};

// Philox4x32-10, the counter-based generator of Salmon, Moraes, Dror and Shaw
// ("Parallel random numbers: as easy as 1, 2, 3", 2011): ten rounds of two
// 32x32-bit products on a 128-bit counter.
__device__ __forceinline__ uint4 philox(uint64_t lo, uint64_t hi, uint64_t key)
{
    uint32_t c0 = (uint32_t)lo, c1 = (uint32_t)(lo >> 32), c2 = (uint32_t)hi, c3 = (uint32_t)(hi >> 32);
    uint32_t k0 = (uint32_t)key, k1 = (uint32_t)(key >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u, k1 += 0xBB67AE85u;
    }
    return uint4{c0, c1, c2, c3};
}
// Which of the eight values of chunk `chunk` of a matrix stay, a bit each.
__device__ __forceinline__ uint32_t kept_of(uint32_t threshold, uint64_t seed, uint64_t offset, uint64_t chunk)
{
    const uint4 w = philox(chunk, offset, seed);
    const uint32_t r[4] = {w.x, w.y, w.z, w.w};
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) bits |= (uint32_t)((i & 1 ? r[i >> 1] >> 16 : r[i >> 1] & 0xFFFFu) >= threshold) << i;
    return bits;
}
// Multiplies or drops the eight values of a chunk.
__device__ __forceinline__ void drop_eight(const Drop &d, uint64_t seed, uint64_t offset, uint64_t chunk, float (&v)[8])
{
    const uint4 w = philox(chunk, offset, seed);
    const uint32_t r[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t bits = i & 1 ? r[i >> 1] >> 16 : r[i >> 1] & 0xFFFFu;
        v[i] = bits < d.threshold ? 0.f : v[i] * d.scale;
    }
}

// ---------------------------------------------------------------------------
// norms
// ---------------------------------------------------------------------------
struct NormOf {
    int32_t kind;  // dbs_norm_kind
    float eps;
    const void *w, *b;  // NULL: ones, zeros
};

// xh = (x f - mean) rstd.  f is 1, or 2^-80 or 2^100 where the squares of a row would
// leave the range of 32 bits above or below.
struct Stat {
    float f, mean, rstd;
    __device__ __forceinline__ float xh(float x) const { return __builtin_fmaf(x, f, -mean) * rstd; }
};
// A row's norm and the two means that its gradient subtracts:
// dx = rstd f (g - xh m1 - m2), m1 the mean of g xh, m2 (layer) that of g.  (With an f above
// 1 rstd f may leave the range of 32 bits where dx does not.)
struct BackStat {
    Stat s;
    float m1, m2;
    __device__ __forceinline__ float dx(float g, float xh) const { return (g - __builtin_fmaf(xh, m1, m2)) * (s.rstd * s.f); }
    __device__ __forceinline__ float dx_any(float g, float xh) const
    {
        return (g - __builtin_fmaf(xh, m1, m2)) * (s.rstd * fminf(s.f, 1.f)) * fmaxf(s.f, 1.f);
    }
};

// stream = scale * res + gate * drop(after(branch)); h = before(stream).
// A norm alone: no branch, h = before(res).
struct EdgeArgs {
    const void *branch, *res;
    int64_t ldb, ldr;
    NormOf after, before;
    const void *gate;
    int64_t ldg;  // 0: one row of gates
    float scale;
    Drop drop;
    void *stream, *h;
    int64_t lds, ldh;
    uint8_t *codes, *exps;  // h as row blocks of 8 bits in place of h
    int32_t rows, n;
};
hipError_t launch_edge(bool bf16, const EdgeArgs &a, int32_t cus, hipStream_t s);

// Gradients.  ds* = ds + the gradient through `before` (at `stream`);
// dres = scale ds*; the rest as the chain rule has it.  A norm alone: no branch,
// stream its input, dres its gradient.
enum { SUM_BEFORE_W, SUM_BEFORE_B, SUM_AFTER_W, SUM_AFTER_B, SUM_GATE, SUMS };
struct EdgeBackArgs {
    const void *ds, *dh, *branch, *stream;
    int64_t ldds, lddh, ldb, lds;
    NormOf after, before;
    const void *gate;
    int64_t ldg;
    float scale;
    Drop drop;
    void *dres, *dbranch, *dgate;  // dgate: of gates by row
    int64_t lddr, lddb, lddg;
    void *sum[SUMS];               // gradients that are sums over the rows, NULL: not wanted
    int32_t rows, n;
    // filled by the launcher
    float *part;                   // [workgroups][sums wanted][n]
    BackStat *stat;                // [rows][before, after], long rows
    int32_t at[SUMS], sums;        // place of a sum among those wanted, -1; their number
    int32_t blocks;                // workgroups along the rows
};
// Bytes of workspace (part, then stat).
size_t edge_back_work(int32_t rows, int32_t n, int sums, int32_t cus);
hipError_t launch_edge_back(bool bf16, EdgeBackArgs a, bool has_branch, void *work, int32_t cus, hipStream_t s);

// out[c] = the sum of part[0 .. blocks - 1][c], in that order.
hipError_t launch_column_total(bool bf16, const float *part, int32_t blocks, int32_t n, void *out, hipStream_t s);

hipError_t launch_dropout(bool bf16, const void *x, int64_t ldx, int32_t rows, int32_t n, const Drop &d, void *y, int64_t ldy,
                          int32_t cus, hipStream_t s);

}  // namespace dbs
