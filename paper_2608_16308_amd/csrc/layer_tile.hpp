// Parts that the tiled matrix products share: the tiles and their places, the
// epilogue, tiles in parts along k.
#pragma once
#include <algorithm>

#include "device_common.hpp"
#include "layer.hpp"

namespace dbs {

constexpr int BK = 64;    // elements of the sum per step
constexpr int GROUP = 4;  // rows of tiles that are worked on together
constexpr int64_t MAX_TILES = 1 << 30;
constexpr double JOIN_STEPS = 2;  // steps that a tile's sums take to memory or back

typedef short s4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u4_t __attribute__((ext_vector_type(4)));

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
    // workgroups that fit the LDS of a compute unit
    static constexpr int per_cu(int stages) { return 160 * 1024 / (stages * (PB + QB)); }
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

// A store at any alignment.
template <class V> struct __attribute__((packed, aligned(1))) Any {
    V v;
};
template <class V> __device__ __forceinline__ void store_any(void *p, V v)
{
    static_assert(alignof(Any<V>) == 1, "a type that cannot be packed");
    ((Any<V> *)p)->v = v;
}

// Rounds and stores a wave's 16 MT x 64 sums (gated: 32 columns of each
// projection): q0 and p0 are its first row and column, z the product of a batch.
template <class X, int KIND, int MT>
__device__ __forceinline__ void epilogue(const GemmArgs &a, const f4_t (&acc)[MT][4], int q0, int p0, int z)
{
    typedef typename X::T T;
    typedef typename X::V8 V8;
    typedef typename X::V4 V4;
    const int lane = lane_id(), r = lane & 15, g = lane >> 4;
    if constexpr ((KIND == G_DX || KIND == G_DW)) {
        T *y = (T *)a.y[z];
        const int64_t ld = a.ldy[z];
        const float scale = a.scale ? *a.scale : 1.f;
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const int row = q0 + 16 * m + r;
            if (row >= a.qn) continue;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int col = p0 + 16 * j + 4 * g;
                T *dst = y + (int64_t)row * ld + col;
                V4 v;
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = (T)(acc[m][j][i] * scale);
                if (col + 4 <= a.pn) store_any(dst, v);
                else
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (col + i < a.pn) dst[i] = v[i];
            }
        }
    } else {
        // a lane's columns: 16 in a row (gated: 8 of gate and the same 8 of up)
        constexpr int NC = KIND == G_GATED ? 8 : 16;
        const int col = p0 + (KIND == G_GATED ? 8 * g : 16 * g);
        // rounds to the element type, keeps v, lanes of a group of 32 columns together
        auto save = [&](const SaveTo &to, const float (&v)[NC], int row) {
            T t[NC];
#pragma unroll
            for (int i = 0; i < NC; ++i) t[i] = (T)v[i];
            if (to.full) {
                if (row >= a.qn) return;
                T *dst = (T *)to.full + (int64_t)row * to.ld + col;
                if (col + NC <= a.pn) {
#pragma unroll
                    for (int i = 0; i < NC; i += 8) {
                        V8 o;
#pragma unroll
                        for (int h = 0; h < 8; ++h) o[h] = t[i + h];
                        store_any(dst + i, o);
                    }
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
            if (col + NC <= a.pn) {
                uint32_t w[NC / 4];
#pragma unroll
                for (int i = 0; i < NC / 4; ++i)
                    w[i] = (uint32_t)(uint8_t)code[4 * i] | (uint32_t)(uint8_t)code[4 * i + 1] << 8 |
                           (uint32_t)(uint8_t)code[4 * i + 2] << 16 | (uint32_t)(uint8_t)code[4 * i + 3] << 24;
                if (NC == 16) store_any(dst, u4_t{w[0], w[1], w[NC / 4 - 2], w[NC / 4 - 1]});
                else store_any(dst, u2_t{w[0], w[1]});
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
            const int row = q0 + 16 * m + r;
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
                act_values(a.act, v);
#pragma unroll
                for (int i = 0; i < NC; ++i) v[i] *= up[i];
            } else {
#pragma unroll
                for (int i = 0; i < NC; ++i) v[i] = acc[m][i >> 2][i & 3] + bias[i];
                if (a.save[0].full || a.save[0].codes) save(a.save[0], v, row);
                act_values(a.act, v);
            }
            if (row >= a.qn || col >= a.pn) continue;
            T *dst = (T *)a.y[0] + (int64_t)row * a.ldy[0] + col;
            const T *res = KIND == G_LINEAR && a.res ? (const T *)a.res + (int64_t)row * a.ldr + col : nullptr;
            if (col + NC <= a.pn) {
#pragma unroll
                for (int h = 0; h < NC; h += 8) {
                    V8 o;
                    if (res) {
                        const V8 add = load_eight<X>(res + h);
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[h + i] += (float)add[i];
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) o[i] = (T)v[h + i];
                    store_any(dst + h, o);
                }
            } else
#pragma unroll
                for (int i = 0; i < NC; ++i)
                    if (col + i < a.pn) dst[i] = (T)(v[i] + (res ? (float)res[i] : 0.f));
        }
    }
}

// What a workgroup does: steps s0 .. s1 - 1 of a tile.
struct Unit {
    int q0, p0, z, s0, s1;
    int tile;  // of those in parts, -1: whole
    int part;
};
// Tiles follow each other in groups of GROUP rows of tiles.
template <int DQ, int DP> __device__ __forceinline__ Unit place_of(const GemmArgs &a, int tile)
{
    Unit u{};
    u.z = tile / (a.tp * a.tq);
    tile -= u.z * a.tp * a.tq;
    const int per = GROUP * a.tp, grp = tile / per, first = grp * GROUP, gsz = min(GROUP, a.tq - first);
    u.q0 = (first + (tile - grp * per) % gsz) * DQ;
    u.p0 = (tile - grp * per) / gsz * DP;
    return u;
}
// The first `full` tiles are taken whole, one round of workgroups after the
// other; the rest, which would leave most compute units idle in the last round,
// in parts along k.  Each XCD has a stretch of neighbouring tiles, for its L2.
template <int DQ, int DP> __device__ __forceinline__ Unit unit_of(const GemmArgs &a)
{
    const int ntile = a.tp * a.tq * a.batch, steps = (a.kn + BK - 1) / BK * a.segs;
    const int id = (int)blockIdx.x + a.first, rest = id >= a.full;
    const int n = rest ? (ntile - a.full) * a.splits : a.full, i = rest ? id - a.full : id;
    const int x = i & 7, each = n >> 3, rem = n & 7;
    const int at = x * each + min(x, rem) + (i >> 3);
    Unit u;
    u.part = rest ? at % a.splits : 0;
    u.tile = rest && a.splits > 1 ? at / a.splits : -1;
    u.s0 = rest ? (int)((int64_t)steps * u.part / a.splits) : 0;
    u.s1 = rest ? (int)((int64_t)steps * (u.part + 1) / a.splits) : steps;
    const Unit at_tile = place_of<DQ, DP>(a, rest ? a.full + at / a.splits : at);
    u.q0 = at_tile.q0, u.p0 = at_tile.p0, u.z = at_tile.z;
    return u;
}

// A tile in parts: each workgroup leaves its sums in memory.
template <int NT, int MT> __device__ __forceinline__ void leave_part(const GemmArgs &a, const Unit &u, const f4_t (&acc)[MT][4])
{
    f4_t *own = (f4_t *)a.part + (int64_t)(u.tile * a.splits + u.part) * MT * 4 * NT + threadIdx.x;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int j = 0; j < 4; ++j) own[(m * 4 + j) * NT] = acc[m][j];
}

// The sums of the tiles in parts, added in the order of the parts; a workgroup
// takes 16 rows of each of a tile's waves.
template <class X, int KIND, int NWQ, int NWP, int MT> static __global__ __launch_bounds__(64 * NWQ * NWP) void k_join(GemmArgs a)
{
    using C = Tile<X, KIND, NWQ, NWP, MT>;
    const int tid = (int)threadIdx.x, wave = wave_id(), wq = wave / NWP, wp = wave % NWP;
    const int tile = (int)blockIdx.x / MT, m = (int)blockIdx.x % MT;
    const Unit u = place_of<C::TQ, KIND == G_GATED ? C::TP / 2 : C::TP>(a, a.full + tile);
    const f4_t *all = (const f4_t *)a.part + ((int64_t)tile * a.splits * MT + m) * 4 * C::NT + tid;
    f4_t acc[1][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[0][j] = all[j * C::NT];
    for (int p = 1; p < a.splits; ++p)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[0][j] += all[((int64_t)p * MT * 4 + j) * C::NT];
    epilogue<X, KIND, 1>(a, acc, u.q0 + 16 * (MT * wq + m), u.p0 + (KIND == G_GATED ? 32 : 64) * wp, u.z);
}
// How many tiles are taken whole and in how many parts the others; the steps
// that a compute unit does in sequence, joining included (a tile's sums are
// written, and those of all its parts read).
static double plan_parts(GemmArgs &a, const LayerWork &w, int64_t ntile, int per_cu, int64_t tile_bytes)
{
    const int64_t slots = (int64_t)w.cus * per_cu, steps = (int64_t)((a.kn + BK - 1) / BK) * a.segs;
    const int64_t rest = ntile % slots;
    a.full = (int32_t)(ntile - rest), a.splits = 1;
    const double whole = (double)(ntile / slots) * (double)steps;
    if (rest == 0) return whole;
    double best = (double)steps;
    for (int64_t s = 2; s <= 16 && s * 2 <= steps && rest * s * tile_bytes <= (int64_t)w.part_bytes; ++s) {
        const double cost = (double)((rest * s + slots - 1) / slots) * (double)((steps + s - 1) / s) + JOIN_STEPS * (1.0 + s);
        if (cost < best) best = cost, a.splits = (int32_t)s;
    }
    return whole + best;
}

// The tiles of a call with a given kernel, `per_cu` workgroups of which fit a
// compute unit; false: too many.
template <class C, int KIND> static bool lay_out(const LayerWork &w, GemmArgs &a, int per_cu, double *steps)
{
    constexpr int DP = KIND == G_GATED ? C::TP / 2 : C::TP;
    const int64_t tq = ((int64_t)a.qn + C::TQ - 1) / C::TQ, tp = ((int64_t)a.pn + DP - 1) / DP, ntile = tq * tp * a.batch;
    if (ntile > MAX_TILES) return false;
    a.tq = (int32_t)tq, a.tp = (int32_t)tp;
    *steps = plan_parts(a, w, ntile, per_cu, (int64_t)C::TP * C::TQ * 4);
    return true;
}

#define LDS_PTR(p) ((__attribute__((address_space(3))) void *)(p))
#define GLB_PTR(p) ((const __attribute__((address_space(1))) void *)(p))

}  // namespace dbs
