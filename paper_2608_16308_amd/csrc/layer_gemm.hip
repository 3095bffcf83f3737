// Matrix products of the dense layer operators on the matrix cores, in tiles
// through LDS, with their epilogues.
#include <algorithm>

#include "device_common.hpp"
#include "layer.hpp"

namespace dbs {

constexpr int BK = 64;  // elements of the sum per step

typedef short s4_t __attribute__((ext_vector_type(4)));

template <class X> struct __attribute__((packed, aligned(2))) Chunk {
    typename X::V8 v;
};

// Eight elements from p, of which the first `left` exist.
template <class X> __device__ __forceinline__ typename X::V8 load_chunk(const typename X::T *p, int64_t left)
{
    if (left >= 8) return ((const Chunk<X> *)p)->v;
    typename X::V8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < left ? p[i] : (typename X::T)0.f;
    return v;
}

// LDS tiles hold 16-byte chunks of eight elements in rows, chunk c of row r at
// place c ^ swz(r), so that the lanes of one read fall into different banks.
//   along k   (rows of the operand are contiguous in k): a tile row is an
//             operand row, 8 chunks of k
//   across k  (the operand is stored k by k): a tile row is one k, TC / 8
//             chunks; ds_read_b64_tr_b16 gives each lane four k of its column
__device__ __forceinline__ int swz_q(int r) { return r & 7; }

template <int KIND> __device__ __forceinline__ int swz_p(int r)
{
    return KIND == G_GATED ? (r & 3) | ((r >> 1) & 4) : (r & 3) | ((r >> 2) & 4);
}
template <int TC> __device__ __forceinline__ int swz_k(int k)
{
    return (((k & 3) | ((k >> 1) & 12)) & (TC / 16 - 1)) << 1;
}

template <class X, int KIND, int NWQ, int NWP, int MT>
struct Tile {
    static constexpr int NT = 64 * NWQ * NWP;
    static constexpr int TQ = NWQ * MT * 16, TP = NWP * 64;
    static constexpr bool PKS = KIND == G_DX || KIND == G_DW, QKS = KIND == G_DW;
    static constexpr int PB = TP * BK * 2, QB = TQ * BK * 2;
    static constexpr int LP = PB / 16 / NT, LQ = QB / 16 / NT;  // chunks per thread and step
    static_assert(PB % (16 * NT) == 0 && QB % (16 * NT) == 0, "whole chunks per thread");
};

// The operand row and matrix of row r of a P tile (along k).
template <int KIND> __device__ __forceinline__ int p_row(int r, int &mat)
{
    if (KIND == G_GATED) {
        mat = (r >> 5) & 1;
        return (r >> 6) * 32 + (r & 31);
    }
    mat = 0;
    return r;
}

template <class X, int KIND, int NWQ, int NWP, int MT>
__global__ __launch_bounds__(64 * NWQ * NWP) void k_tile(GemmArgs a)
{
    using C = Tile<X, KIND, NWQ, NWP, MT>;
    typedef typename X::T T;
    typedef typename X::V8 V8;
    typedef typename X::V4 V4;
    __shared__ __attribute__((aligned(16))) uint8_t lds[2][C::PB + C::QB];
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = wave_id();
    const int wq = wave / NWP, wp = wave % NWP, r = lane & 15, g = lane >> 4;

    // tiles in groups of 8 rows of tiles, each XCD a stretch of its own
    const int ntile = a.tp * a.tq, total = ntile * a.splits;
    int id = (int)blockIdx.x;
    {
        const int x = id & 7, qn = total >> 3, rem = total & 7;
        id = x * qn + (x < rem ? x : rem) + (id >> 3);
    }
    const int tile = id / a.splits, split = id - tile * a.splits;
    const int per = 8 * a.tp, grp = tile / per, first = grp * 8, gsz = min(8, a.tq - first);
    const int tqi = first + (tile - grp * per) % gsz, tpi = (tile - grp * per) / gsz;
    const int z = (int)blockIdx.y;
    const int q0 = tqi * C::TQ;
    const int p0 = tpi * (KIND == G_GATED ? C::TP / 2 : C::TP);

    const int ksteps = (a.kn + BK - 1) / BK, steps = ksteps * a.segs;
    const int s0 = (int)((int64_t)steps * split / a.splits), s1 = (int)((int64_t)steps * (split + 1) / a.splits);

    V8 rp[C::LP], rq[C::LQ];
    auto fetch = [&](int step) {
        const int seg = a.segs > 1 && step >= ksteps ? 1 : 0;
        const int k0 = (step - seg * ksteps) * BK;
#pragma unroll
        for (int i = 0; i < C::LP; ++i) {
            const int c = i * C::NT + tid;
            if constexpr (C::PKS) {
                const int k = c / (C::TP / 8), col = p0 + 8 * ((c % (C::TP / 8)) ^ swz_k<C::TP>(k));
                const int left = k0 + k < a.kn ? a.pn - col : 0;
                rp[i] = load_chunk<X>((const T *)a.p[seg] + (int64_t)(k0 + k) * a.ldp[seg] + col, left);
            } else {
                int mat;
                const int row = p0 + p_row<KIND>(c >> 3, mat), k = k0 + 8 * ((c & 7) ^ swz_p<KIND>(c >> 3));
                rp[i] = load_chunk<X>((const T *)a.p[mat] + (int64_t)row * a.ldp[mat] + k, row < a.pn ? a.kn - k : 0);
            }
        }
#pragma unroll
        for (int i = 0; i < C::LQ; ++i) {
            const int c = i * C::NT + tid;
            if constexpr (C::QKS) {
                const int k = c / (C::TQ / 8), col = q0 + 8 * ((c % (C::TQ / 8)) ^ swz_k<C::TQ>(k));
                rq[i] = load_chunk<X>((const T *)a.q[z] + (int64_t)(k0 + k) * a.ldq[z] + col,
                                      k0 + k < a.kn ? a.qn - col : 0);
            } else {
                const int row = q0 + (c >> 3), k = k0 + 8 * ((c & 7) ^ swz_q(c >> 3));
                rq[i] = load_chunk<X>((const T *)a.q[seg] + (int64_t)row * a.ldq[seg] + k, row < a.qn ? a.kn - k : 0);
            }
        }
    };
    auto stage = [&](int buf) {
#pragma unroll
        for (int i = 0; i < C::LP; ++i) *(V8 *)(lds[buf] + (i * C::NT + tid) * 16) = rp[i];
#pragma unroll
        for (int i = 0; i < C::LQ; ++i) *(V8 *)(lds[buf] + C::PB + (i * C::NT + tid) * 16) = rq[i];
    };

    f4_t acc[MT][4];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[m][j] = f4_t{0.f, 0.f, 0.f, 0.f};

    // read four k of a column (across k): lane s4 = r / 4 of a group of 16
    // gives the address of k = s4, columns 4 (r % 4) .. + 3
    auto tr = [&](const uint8_t *p) {
        return __builtin_bit_cast(V4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4_t *)p));
    };
    auto across = [&](const uint8_t *base, int tcols, int swz, int s, int unit) {
        const int k = 32 * s + 8 * g + (r >> 2);
        const uint8_t *p = base + k * tcols * 2 + (((unit << 1) ^ swz) + ((r >> 1) & 1)) * 16 + (r & 1) * 8;
        const V4 lo = tr(p), hi = tr(p + 4 * tcols * 2);
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    auto compute = [&](int buf) {
        const uint8_t *lp = lds[buf], *lq = lds[buf] + C::PB;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            V8 fp[4], fq[MT];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (C::PKS) fp[j] = across(lp, C::TP, swz_k<C::TP>(8 * g + (r >> 2)), s, 4 * wp + j);
                else {
                    const int row = KIND == G_GATED ? 64 * wp + 32 * (j >> 1) + 8 * (r >> 2) + 4 * (j & 1) + (r & 3)
                                                    : 64 * wp + 16 * (r >> 2) + 4 * j + (r & 3);
                    fp[j] = *(const V8 *)(lp + row * 128 + ((4 * s + g) ^ swz_p<KIND>(row)) * 16);
                }
            }
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                if constexpr (C::QKS) fq[m] = across(lq, C::TQ, swz_k<C::TQ>(8 * g + (r >> 2)), s, MT * wq + m);
                else {
                    const int row = 16 * (MT * wq + m) + r;
                    fq[m] = *(const V8 *)(lq + row * 128 + ((4 * s + g) ^ swz_q(row)) * 16);
                }
            }
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[m][j] = X::mma(fp[j], fq[m], acc[m][j]);
        }
    };

    if (s0 < s1) {
        fetch(s0);
        stage(0);
    }
    for (int t = s0; t < s1; ++t) {
        const int buf = (t - s0) & 1;
        __syncthreads();
        if (t + 1 < s1) fetch(t + 1);
        compute(buf);
        if (t + 1 < s1) stage(buf ^ 1);
    }

    // ---- epilogue
    if constexpr (C::PKS) {
        T *y = (T *)a.y[z];
        const int64_t ld = a.ldy[z];
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const int row = q0 + 16 * (MT * wq + m) + r;
            if (row >= a.qn) continue;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int col = p0 + 64 * wp + 16 * j + 4 * g;
                T *dst = y + (int64_t)row * ld + col;
                V4 v;
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = (T)acc[m][j][i];
                if (a.vec && col + 4 <= a.pn) *(V4 *)dst = v;
                else
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (col + i < a.pn) dst[i] = v[i];
            }
        }
    } else {
        // a lane's columns: 16 in a row (gated: 8 of gate and the same 8 of up)
        constexpr int NC = KIND == G_GATED ? 8 : 16;
        const int col = p0 + (KIND == G_GATED ? 32 * wp + 8 * g : 64 * wp + 16 * g);
        // rounds to the element type, keeps v, lanes of a group of 32 columns together
        auto save = [&](const SaveTo &to, const float (&v)[NC], int row) {
            T t[NC];
#pragma unroll
            for (int i = 0; i < NC; ++i) t[i] = (T)v[i];
            if (to.full) {
                if (row >= a.qn) return;
                T *dst = (T *)to.full + (int64_t)row * to.ld + col;
                if (to.vec && col + NC <= a.pn) {
#pragma unroll
                    for (int i = 0; i < NC; i += 8) *(V8 *)(dst + i) = *(const V8 *)(t + i);
                } else
#pragma unroll
                    for (int i = 0; i < NC; ++i)
                        if (col + i < a.pn) dst[i] = t[i];
                return;
            }
            float big = 0.f;
#pragma unroll
            for (int i = 0; i < NC; ++i) big = fmaxf(big, col + i < a.pn ? ck_mag((float)t[i]) : 0.f);
            big = fmaxf(big, __shfl_xor(big, 16, 64));
            if (NC == 8) big = fmaxf(big, __shfl_xor(big, 32, 64));
            if (row >= a.qn || col >= a.pn) return;
            const int e = ck_exp<X>(big);
            const int64_t ngroup = (a.pn + CK_GROUP - 1) / CK_GROUP;
            if (col % CK_GROUP == 0) to.exps[row * ngroup + col / CK_GROUP] = (uint8_t)(e + CK_BIAS);
            int8_t *dst = to.codes + (int64_t)row * a.pn + col;
            int8_t code[NC];
#pragma unroll
            for (int i = 0; i < NC; ++i) code[i] = (int8_t)ck_code((float)t[i], e);
            if (to.vec && col + NC <= a.pn) {
                uint32_t w[NC / 4];
#pragma unroll
                for (int i = 0; i < NC / 4; ++i)
                    w[i] = (uint32_t)(uint8_t)code[4 * i] | (uint32_t)(uint8_t)code[4 * i + 1] << 8 |
                           (uint32_t)(uint8_t)code[4 * i + 2] << 16 | (uint32_t)(uint8_t)code[4 * i + 3] << 24;
                if (NC == 16) *(uint4 *)dst = make_uint4(w[0], w[1], w[NC / 4 - 2], w[NC / 4 - 1]);
                else *(uint2 *)dst = make_uint2(w[0], w[1]);
            } else
#pragma unroll
                for (int i = 0; i < NC; ++i)
                    if (col + i < a.pn) dst[i] = code[i];
        };
        float bias[NC];
        if constexpr (KIND == G_LINEAR) {
#pragma unroll
            for (int i = 0; i < NC; ++i) bias[i] = a.bias && col + i < a.pn ? (float)((const T *)a.bias)[col + i] : 0.f;
        }
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const int row = q0 + 16 * (MT * wq + m) + r;
            float v[NC];
            if constexpr (KIND == G_GATED) {
                float up[NC];
#pragma unroll
                for (int i = 0; i < NC; ++i) {
                    v[i] = acc[m][i >> 2][i & 3];
                    up[i] = acc[m][2 + (i >> 2)][i & 3];
                }
                if (a.save[0].full || a.save[0].codes) {
                    save(a.save[0], v, row);
                    save(a.save[1], up, row);
                }
#pragma unroll
                for (int i = 0; i < NC; ++i) v[i] = act_value(a.act, v[i]) * up[i];
            } else {
#pragma unroll
                for (int i = 0; i < NC; ++i) v[i] = acc[m][i >> 2][i & 3] + bias[i];
                if (a.save[0].full || a.save[0].codes) save(a.save[0], v, row);
#pragma unroll
                for (int i = 0; i < NC; ++i) v[i] = act_value(a.act, v[i]);
            }
            if (row >= a.qn || col >= a.pn) continue;
            T *dst = (T *)a.y[0] + (int64_t)row * a.ldy[0] + col;
            const T *res = KIND == G_LINEAR && a.res ? (const T *)a.res + (int64_t)row * a.ldr + col : nullptr;
            if (a.vec && col + NC <= a.pn) {
#pragma unroll
                for (int h = 0; h < NC; h += 8) {
                    V8 o;
                    if (res) {
                        const V8 add = *(const V8 *)(res + h);
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[h + i] += (float)add[i];
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) o[i] = (T)v[h + i];
                    *(V8 *)(dst + h) = o;
                }
            } else
#pragma unroll
                for (int i = 0; i < NC; ++i)
                    if (col + i < a.pn) dst[i] = (T)(v[i] + (res ? (float)res[i] : 0.f));
        }
    }
}

template <class X, int KIND, int NWQ, int NWP, int MT> hipError_t launch_tile(GemmArgs a, hipStream_t s)
{
    using C = Tile<X, KIND, NWQ, NWP, MT>;
    a.tq = (a.qn + C::TQ - 1) / C::TQ;
    a.tp = KIND == G_GATED ? (a.pn + C::TP / 2 - 1) / (C::TP / 2) : (a.pn + C::TP - 1) / C::TP;
    a.splits = 1;
    if (a.tq == 0 || a.tp == 0) return hipSuccess;
    hipLaunchKernelGGL((k_tile<X, KIND, NWQ, NWP, MT>), dim3((unsigned)(a.tp * a.tq), (unsigned)a.batch), dim3(C::NT), 0,
                       s, a);
    return hipGetLastError();
}

template <class X> hipError_t launch_kind(GemmKind kind, const GemmArgs &a, hipStream_t s)
{
    switch (kind) {
    case G_LINEAR: return launch_tile<X, G_LINEAR, 2, 2, 4>(a, s);
    case G_GATED: return launch_tile<X, G_GATED, 2, 2, 4>(a, s);
    case G_DX: return launch_tile<X, G_DX, 2, 2, 4>(a, s);
    default: return launch_tile<X, G_DW, 2, 2, 4>(a, s);
    }
}

hipError_t launch_gemm(const LayerWork &w, bool bf16, GemmKind kind, GemmArgs a, hipStream_t s)
{
    (void)w;
    return bf16 ? launch_kind<Bf16>(kind, a, s) : launch_kind<Fp16>(kind, a, s);
}

}  // namespace dbs
