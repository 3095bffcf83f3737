// The forward products for a few tokens: the weights are read once, straight
// into registers, by workgroups that each take 16 rows of them.
#include <algorithm>

#include "device_common.hpp"
#include "layer.hpp"

namespace dbs {

// (weights pass once: they need not stay in the caches)
template <class X> __device__ __forceinline__ typename X::V8 load_once(const typename X::T *p)
{
    typedef typename X::V8 V8u __attribute__((aligned(2)));
    return __builtin_nontemporal_load((const V8u *)p);
}
// Keeps a projection of token t, a column a lane: in 16 bits, or in 8, where 32
// neighbouring lanes hold the columns of a group (`in`: one that exists).
template <class X>
__device__ __forceinline__ void keep_one(const SaveTo &to, float v, bool in, int t, int col, int cols, int64_t ngroup)
{
    typedef typename X::T T;
    const T q = (T)v;
    if (to.full) {
        if (in) ((T *)to.full)[(int64_t)t * to.ld + col] = q;
    } else if (to.codes) {
        float big = in ? ck_mag((float)q) : 0.f;
#pragma unroll
        for (int o = 1; o < CK_GROUP; o <<= 1) big = fmaxf(big, __shfl_xor(big, o, 64));
        if (!in) return;
        const int e = ck_exp<X>(big);
        to.codes[(int64_t)t * cols + col] = (int8_t)ck_code((float)q, e);
        if (col % CK_GROUP == 0) to.exps[t * ngroup + col / CK_GROUP] = (uint8_t)(e + CK_BIAS);
    }
}

// A column of token t from its sum (gated: of both projections).
template <class X, bool GATED>
__device__ __forceinline__ void finish_one(const GemmArgs &a, float sum, float up, bool in, int t, int col, int64_t ngroup)
{
    typedef typename X::T T;
    float v[1] = {sum};
    if (!GATED && a.bias && in) v[0] += (float)((const T *)a.bias)[col];
    keep_one<X>(a.save[0], v[0], in, t, col, a.pn, ngroup);
    if (GATED) keep_one<X>(a.save[1], up, in, t, col, a.pn, ngroup);
    act_values(a.act, v);
    if (GATED) v[0] *= up;
    else if (a.res && in) v[0] += (float)((const T *)a.res)[(int64_t)t * a.ldr + col];
    if (in) ((T *)a.y[0])[(int64_t)t * a.ldy[0] + col] = (T)v[0];
}

constexpr int RW_U = 8;                // products of 32 k in a wave's turn
constexpr int RW_K = 32 * RW_U;
constexpr int RW_MAX_WAVES = 8;
constexpr int RW_ROW = RW_K * 2 + 16;  // bytes of a row in LDS: 16 rows start in different banks

// A wave multiplies 16 rows of w (gated: 8 of either matrix) with up to 16
// tokens over its turns of RW_K elements; the waves' sums are added in LDS, in
// their order.  A workgroup does `groups` times 16 rows, one after the other (32
// columns, a group of a checkpoint, where one is kept).  Rows and tokens past the
// last are read as the last one, and not written.
//
// Loads follow the rows, 512 bytes of two rows an instruction, and a bounce
// through LDS that is private to the wave brings them to the operands' order;
// those of the next turn are on their way while one is multiplied.
template <class X, bool GATED>
__global__ __launch_bounds__(64 * RW_MAX_WAVES, 3) void k_rows_dense(GemmArgs a, int groups)
{
    typedef typename X::T T;
    typedef typename X::V8 V8;
    constexpr int COLS = GATED ? 8 : 16;  // of a group of rows
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const int lane = lane_id(), wave = wave_id(), waves = (int)blockDim.x / 64, r = lane & 15, g = lane >> 4;
    const int half = lane >> 5, at = 8 * (lane & 31);
    uint8_t *lw = lds + wave * (16 + a.qn) * RW_ROW, *lx = lw + 16 * RW_ROW;
    const uint8_t *rw = lw + r * RW_ROW + 16 * g, *rx = lx + min(r, a.qn - 1) * RW_ROW + 16 * g;
    float *sums = (float *)lds, *total = sums + max(waves * 256, waves * (16 + a.qn) * (RW_ROW / 4));
    // rows of x, in elements from the first
    uint32_t ox[8];
#pragma unroll
    for (int t = 0; t < 8; ++t) ox[t] = (uint32_t)min(2 * t + half, a.qn - 1) * (uint32_t)a.ldq[0] + at;
    const T *x = (const T *)a.q[0];
    const int block = (int)blockIdx.x + a.first;

    for (int n = 0; n < groups; ++n) {
        // (a checkpoint's last group of columns may have no rows left)
        const int p0 = min((block * groups + n) * COLS, a.pn - 1);
        // rows of w, from the first of their matrix
        const T *w[2];
        uint32_t ow[8];
#pragma unroll
        for (int m = 0; m < (GATED ? 2 : 1); ++m) w[m] = (const T *)a.p[m] + (int64_t)p0 * a.ldp[m];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int row = 2 * i + half, m = 2 * i / COLS;
            ow[i] = (uint32_t)min(row % COLS, a.pn - 1 - p0) * (uint32_t)a.ldp[m] + at;
        }
        V8 vw[8], vx[8];
        auto fetch = [&](int k) {
#pragma unroll
            for (int t = 0; t < 8; ++t)
                if (2 * t < a.qn) vx[t] = load_eight<X>(x + k + ox[t]);
#pragma unroll
            for (int i = 0; i < 8; ++i) vw[i] = load_once<X>(w[2 * i / COLS] + k + ow[i]);
        };
        f4_t acc = {0.f, 0.f, 0.f, 0.f};
        auto multiply = [&]() {
            wave_lds_sync();
#pragma unroll
            for (int u = 0; u < RW_U; ++u) {
                acc = X::mma(*(const V8 *)(rw + 64 * u), *(const V8 *)(rx + 64 * u), acc);
                if (u % 4 == 3) __builtin_amdgcn_sched_barrier(0);  // (registers for the loads in flight)
            }
            wave_lds_sync();
        };
        int k = wave * RW_K;
        if (k + RW_K <= a.kn) fetch(k);
        for (; k + RW_K <= a.kn; k += waves * RW_K) {
#pragma unroll
            for (int t = 0; t < 8; ++t)
                if (2 * t + half < a.qn) *(V8 *)(lx + (2 * t + half) * RW_ROW + 2 * at) = vx[t];
#pragma unroll
            for (int i = 0; i < 8; ++i) *(V8 *)(lw + (2 * i + half) * RW_ROW + 2 * at) = vw[i];
            const int next = k + waves * RW_K;
            if (next + RW_K <= a.kn) fetch(next);
            multiply();
        }
        if (k < a.kn) {  // the last turn, ragged
#pragma unroll 4
            for (int t = 0; 2 * t < a.qn; ++t) {
                const int row = min(2 * t + half, a.qn - 1);
                *(V8 *)(lx + row * RW_ROW + 2 * at) = load_end<X>(x + (int64_t)row * a.ldq[0], k + at, a.kn);
            }
#pragma unroll 4
            for (int i = 0; i < 8; ++i) {
                const int row = 2 * i + half, m = 2 * i / COLS;
                *(V8 *)(lw + row * RW_ROW + 2 * at) =
                    load_end<X>((const T *)a.p[m] + (int64_t)min(p0 + row % COLS, a.pn - 1) * a.ldp[m], k + at, a.kn);
            }
            multiply();
        }
        __syncthreads();
        // lane (g, r) holds rows 4 g .. + 3 of w for token r
#pragma unroll
        for (int i = 0; i < 4; ++i) sums[(wave * 4 + i) * 64 + lane] = acc[i];
        __syncthreads();
        for (int c = (int)threadIdx.x; c < 256; c += (int)blockDim.x) {
            float s = sums[c];
            for (int v = 1; v < waves; ++v) s += sums[v * 256 + c];
            // c = 64 i + 16 g + r: row 4 g + i of token r
            total[(n * 16 + (c & 15)) * 16 + 4 * ((c >> 4) & 3) + (c >> 6)] = s;
        }
        __syncthreads();
    }
    // a thread per token and column, a row of columns in neighbouring lanes
    const int cols = COLS * groups;
    const int64_t ngroup = (a.pn + CK_GROUP - 1) / CK_GROUP;
    for (int c = (int)threadIdx.x; c < 16 * cols; c += (int)blockDim.x) {
        const int token = c / cols, cc = c % cols, col = block * cols + cc;
        const bool in = token < a.qn && col < a.pn;
        const float *of = total + ((cc / COLS) * 16 + token) * 16 + cc % COLS;
        finish_one<X, GATED>(a, of[0], GATED ? of[8] : 0.f, in, token, col, ngroup);
    }
}

// Waves of a workgroup: as many as fill the device (each has 8 KB and more in
// flight), with turns that they share out evenly where that costs less than
// half of them.  What is kept does not matter here, so that it does not change
// the order of a sum.
static int waves_of(const LayerWork &w, int64_t groups, int64_t kn)
{
    const int64_t turns = (kn + RW_K - 1) / RW_K, fill = (16 * (int64_t)w.cus + groups - 1) / groups;
    const int64_t most = std::max<int64_t>(1, std::min<int64_t>({turns, std::max<int64_t>(fill, 4), RW_MAX_WAVES}));
    int64_t best = most;
    for (int64_t n = most; 2 * n >= most; --n)
        if ((turns + n - 1) / n * n < (turns + best - 1) / best * best) best = n;
    return (int)best;
}

template <class X, bool GATED> static hipError_t rows_t(const LayerWork &w, GemmArgs a, hipStream_t s)
{
    constexpr int COLS = GATED ? 8 : 16;
    const int64_t groups = ((int64_t)a.pn + COLS - 1) / COLS;
    const int waves = waves_of(w, groups, a.kn), each = a.save[0].codes ? CK_GROUP / COLS : 1;
    const size_t lds = (size_t)std::max(waves * 1024, waves * (16 + a.qn) * RW_ROW) + each * 1024;
    return launch_parts((groups + each - 1) / each, 64 * waves, [&](int32_t first, dim3 grid) {
        a.first = first;
        hipLaunchKernelGGL((k_rows_dense<X, GATED>), grid, dim3((unsigned)(64 * waves)), lds, s, a, each);
    });
}

// ---------------------------------------------------------------------------
// one token
// ---------------------------------------------------------------------------
constexpr int DT_WAVES = 8, DT_CHUNKS = 4, DT_TURN = 512 * DT_CHUNKS;

// A wave takes two rows of w (gated: one of either matrix) and reads them along
// their length, 1 KB an instruction; with few rows, `ks` waves share a pair's
// turns.  A workgroup does `pairs` pairs, one after the other where they are
// more than its waves (32 columns, a group, where a checkpoint is kept).
// Products in 32 bits on the vector ALUs, which have room for it.
template <class X, bool GATED>
__global__ __launch_bounds__(64 * DT_WAVES) void k_rows_dot(GemmArgs a, int ks, int pairs)
{
    typedef typename X::T T;
    typedef typename X::V8 V8;
    __shared__ float sums[CK_GROUP * DT_WAVES][2];  // a row per pair and wave on it
    const int lane = lane_id(), wave = wave_id(), at = 8 * lane, block = (int)blockIdx.x + a.first;
    const T *w[2], *x = (const T *)a.q[0];
    auto add = [&](V8 vw, V8 vx, float &s) {
#pragma unroll
        for (int i = 0; i < 8; ++i) s = __builtin_fmaf((float)vw[i], (float)vx[i], s);
    };
    for (int pair = wave / ks; pair < pairs; pair += DT_WAVES / ks) {
        const int first = block * pairs + pair;
#pragma unroll
        for (int n = 0; n < 2; ++n)
            w[n] = (const T *)a.p[GATED ? n : 0] + (int64_t)min(GATED ? first : 2 * first + n, a.pn - 1) * a.ldp[GATED ? n : 0];
        float acc[2] = {0.f, 0.f};
        int k = (wave % ks) * DT_TURN;
        for (; k + DT_TURN <= a.kn; k += ks * DT_TURN) {
            V8 vw[2][DT_CHUNKS], vx[DT_CHUNKS];
#pragma unroll
            for (int c = 0; c < DT_CHUNKS; ++c)
#pragma unroll
                for (int n = 0; n < 2; ++n) vw[n][c] = load_once<X>(w[n] + k + 512 * c + at);
#pragma unroll
            for (int c = 0; c < DT_CHUNKS; ++c) vx[c] = load_eight<X>(x + k + 512 * c + at);
#pragma unroll
            for (int c = 0; c < DT_CHUNKS; ++c)
#pragma unroll
                for (int n = 0; n < 2; ++n) add(vw[n][c], vx[c], acc[n]);
        }
        for (int c = 0; c < DT_CHUNKS && k + 512 * c < a.kn; ++c) {  // the last turn, ragged
            V8 vw[2];
#pragma unroll
            for (int n = 0; n < 2; ++n) vw[n] = load_end<X>(w[n], k + 512 * c + at, a.kn);
            const V8 vx = load_end<X>(x, k + 512 * c + at, a.kn);
#pragma unroll
            for (int n = 0; n < 2; ++n) add(vw[n], vx, acc[n]);
        }
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const float s = wave_sum(acc[n]);
            if (lane == 0) sums[pair * ks + wave % ks][n] = s;
        }
    }
    __syncthreads();
    // a lane per column
    const int cols = GATED ? pairs : 2 * pairs, c = (int)threadIdx.x, col = block * cols + c;
    if (c >= cols) return;
    auto value = [&](int n) {
        const float(*p)[2] = sums + (GATED ? c : c / 2) * ks;
        float s = p[0][n];
        for (int i = 1; i < ks; ++i) s += p[i][n];
        return s;
    };
    finish_one<X, GATED>(a, value(GATED ? 0 : c % 2), GATED ? value(1) : 0.f, col < a.pn, 0, col,
                         (a.pn + CK_GROUP - 1) / CK_GROUP);
}

template <class X, bool GATED> static hipError_t dot_t(const LayerWork &w, GemmArgs a, hipStream_t s)
{
    const int64_t pairs = GATED ? a.pn : ((int64_t)a.pn + 1) / 2, turns = ((int64_t)a.kn + DT_TURN - 1) / DT_TURN;
    int ks = 1;
    while (ks < DT_WAVES && 2 * ks <= turns && pairs * ks < 8 * (int64_t)w.cus) ks *= 2;
    const int per = a.save[0].codes ? CK_GROUP / (GATED ? 1 : 2) : DT_WAVES / ks;
    return launch_parts((pairs + per - 1) / per, 64 * DT_WAVES, [&](int32_t first, dim3 grid) {
        a.first = first;
        hipLaunchKernelGGL((k_rows_dot<X, GATED>), grid, dim3(64 * DT_WAVES), 0, s, a, ks, per);
    });
}

template <class X, bool GATED> static hipError_t rows_g(const LayerWork &w, const GemmArgs &a, hipStream_t s)
{
    return a.qn == 1 ? dot_t<X, GATED>(w, a, s) : rows_t<X, GATED>(w, a, s);
}

bool rows_take(bool gated, const GemmArgs &a)
{
    const int64_t far = std::max({a.ldq[0], a.ldp[0], gated ? a.ldp[1] : 0});
    return a.qn >= 1 && a.qn <= ROWS_TOKENS && a.kn >= 8 && far <= 1 << 27;
}

hipError_t launch_rows(const LayerWork &w, bool bf16, bool gated, const GemmArgs &a, hipStream_t s)
{
    if (a.pn == 0) return hipSuccess;
    if (gated) return bf16 ? rows_g<Bf16, true>(w, a, s) : rows_g<Fp16, true>(w, a, s);
    return bf16 ? rows_g<Bf16, false>(w, a, s) : rows_g<Fp16, false>(w, a, s);
}

}  // namespace dbs
