// Matrix products of the dense layer operators on the matrix cores, in tiles
// through LDS, with their epilogues.
#include <type_traits>

#include "layer_tile.hpp"

namespace dbs {

// A tile of the product whose operands may stand anywhere: chunks come through
// registers, PF steps ahead, since loads straight into LDS need whole 16-byte
// chunks.  Bound by the edge handling and the wait of one barrier a step.  fp16
// rows of odd length, all compute units at it: forward 650 to 730 TFLOP/s
// (1531x7001->5003, 4096x4097->4096), across k 420 to 460; 777x1111->2003, which
// has few steps, 137 and 90.
template <class X, int KIND, int NWQ, int NWP, int MT, int PF>
__global__ __launch_bounds__(64 * NWQ * NWP, 2) void k_tile(GemmArgs a)
{
    using C = Tile<X, KIND, NWQ, NWP, MT>;
    typedef typename X::T T;
    typedef typename X::V8 V8;
    typedef typename X::V4 V4;
    __shared__ __attribute__((aligned(16))) uint8_t lds[2][C::PB + C::QB];
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = wave_id();
    const int wq = wave / NWP, wp = wave % NWP, r = lane & 15, g = lane >> 4;

    const Unit u = unit_of<C::TQ, KIND == G_GATED ? C::TP / 2 : C::TP>(a);
    const int q0 = u.q0, p0 = u.p0, z = u.z, s0 = u.s0, s1 = u.s1;
    const int ksteps = (a.kn + BK - 1) / BK;

    V8 rp[PF][C::LP], rq[PF][C::LQ];
    // A chunk: elements `at` .. + 7 of row `row` of a matrix of `rows` rows of n
    // elements.  EDGE: it may pass a row's end, and reads as zeros there; else
    // only the rows may be past the last, and are read as the last.
    auto chunk = [&](auto edge, const T *m, int64_t ld, int row, int rows, int at, int n) {
        const T *p = m + (int64_t)min(row, rows - 1) * ld;
        if (!decltype(edge)::value) return load_eight<X>(p + at);
        if (n >= 8) return load_end<X>(p, at, n);
        V8 v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = at + i < n ? p[min(at + i, n - 1)] : (T)0.f;
        return v;
    };
    auto fetch_p = [&](auto edge, int seg, int k0, V8(&v)[C::LP]) {
#pragma unroll
        for (int i = 0; i < C::LP; ++i) {
            const int c = i * C::NT + tid;
            if constexpr (C::PKS) {
                const int k = c / (C::TP / 8), col = p0 + 8 * ((c % (C::TP / 8)) ^ swz_k<C::TP>(k));
                v[i] = chunk(edge, (const T *)a.p[seg], a.ldp[seg], k0 + k, a.kn, col, a.pn);
                if (k0 + k >= a.kn) v[i] = V8{};
            } else {
                int mat;
                const int row = p0 + p_row<KIND>(c >> 3, mat), k = k0 + 8 * ((c & 7) ^ swz_p<KIND>(c >> 3));
                v[i] = chunk(edge, (const T *)a.p[mat], a.ldp[mat], row, a.pn, k, a.kn);
            }
        }
    };
    auto fetch_q = [&](auto edge, int seg, int k0, V8(&v)[C::LQ]) {
#pragma unroll
        for (int i = 0; i < C::LQ; ++i) {
            const int c = i * C::NT + tid;
            if constexpr (C::QKS) {
                const int k = c / (C::TQ / 8), col = q0 + 8 * ((c % (C::TQ / 8)) ^ swz_k<C::TQ>(k));
                v[i] = chunk(edge, (const T *)a.q[z], a.ldq[z], k0 + k, a.kn, col, a.qn);
                if (k0 + k >= a.kn) v[i] = V8{};
            } else {
                const int row = q0 + (c >> 3), k = k0 + 8 * ((c & 7) ^ swz_q(c >> 3));
                v[i] = chunk(edge, (const T *)a.q[seg], a.ldq[seg], row, a.qn, k, a.kn);
            }
        }
    };
    auto fetch = [&](int step, int f) {
        const int seg = a.segs > 1 && step >= ksteps ? 1 : 0;
        const int k0 = (step - seg * ksteps) * BK;
        if (C::PKS ? p0 + C::TP > a.pn : k0 + BK > a.kn) fetch_p(std::true_type{}, seg, k0, rp[f]);
        else fetch_p(std::false_type{}, seg, k0, rp[f]);
        if (C::QKS ? q0 + C::TQ > a.qn : k0 + BK > a.kn) fetch_q(std::true_type{}, seg, k0, rq[f]);
        else fetch_q(std::false_type{}, seg, k0, rq[f]);
    };
    auto stage = [&](int f, int buf) {
#pragma unroll
        for (int i = 0; i < C::LP; ++i) *(V8 *)(lds[buf] + (i * C::NT + tid) * 16) = rp[f][i];
#pragma unroll
        for (int i = 0; i < C::LQ; ++i) *(V8 *)(lds[buf] + C::PB + (i * C::NT + tid) * 16) = rq[f][i];
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

    // PF steps are on their way in registers while one is multiplied
#pragma unroll
    for (int f = 0; f < PF; ++f)
        if (s0 + f < s1) fetch(s0 + f, f);
    for (int t = s0; t < s1;) {
#pragma unroll
        for (int f = 0; f < PF; ++f, ++t) {
            if (t >= s1) break;
            const int buf = (t - s0) & 1;
            stage(f, buf);
            __syncthreads();
            if (t + PF < s1) fetch(t + PF, f);
            compute(buf);
        }
    }

    if (u.tile >= 0) leave_part<C::NT, MT>(a, u, acc);
    else epilogue<X, KIND, MT>(a, acc, q0 + 16 * MT * wq, p0 + (KIND == G_GATED ? 32 : 64) * wp, z);
}


// A tile of the product whose operands are made of whole 16-byte chunks, which
// go straight into LDS, NS steps deep.  The fragments of a half step are read
// while the other half is multiplied.  The 256x256 tile gives each byte of LDS the
// most products; the smaller tiles with three and four stages serve products with
// too few large ones.  Bound by the reads of LDS beside the products, and with two
// stages by the wait for a whole step's loads: the matrix cores are busy 47 to 58%
// of the time (gated 4096x4096->11008 bf16 keeping 8 bits: 694 us, 1060 TFLOP/s).
template <class X, int KIND, int NWQ, int NWP, int MT, int NS>
__global__ __launch_bounds__(64 * NWQ * NWP, 2) void k_block(GemmArgs a)
{
    using C = Tile<X, KIND, NWQ, NWP, MT>;
    typedef typename X::V8 V8;
    typedef typename X::V4 V4;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[NS][C::PB + C::QB];
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = wave_id();
    const int wq = wave / NWP, wp = wave % NWP, r = lane & 15, g = lane >> 4;

    const Unit u = unit_of<C::TQ, KIND == G_GATED ? C::TP / 2 : C::TP>(a);
    const int q0 = u.q0, p0 = u.p0, z = u.z, s0 = u.s0, s1 = u.s1;
    const int ksteps = (a.kn + BK - 1) / BK;

    // where a thread's chunks are, in bytes from the tile's first element of a step
    uint32_t vp[C::LP], vq[C::LQ];
#pragma unroll
    for (int i = 0; i < C::LP; ++i) {
        const int c = i * C::NT + tid;
        if constexpr (C::PKS) {
            const int k = c / (C::TP / 8), col = 8 * ((c % (C::TP / 8)) ^ swz_k<C::TP>(k));
            vp[i] = (uint32_t)(k * (int)a.ldp[0] + min(col, (a.pn - 1 - p0) & ~7)) * 2u;
        } else {
            int mat;
            const int row = p_row<KIND>(c >> 3, mat);
            vp[i] = (uint32_t)(min(row, a.pn - 1 - p0) * (int)a.ldp[mat] + 8 * ((c & 7) ^ swz_p<KIND>(c >> 3))) * 2u;
        }
    }
#pragma unroll
    for (int i = 0; i < C::LQ; ++i) {
        const int c = i * C::NT + tid;
        if constexpr (C::QKS) {
            const int k = c / (C::TQ / 8), col = 8 * ((c % (C::TQ / 8)) ^ swz_k<C::TQ>(k));
            vq[i] = (uint32_t)(k * (int)a.ldq[0] + min(col, (a.qn - 1 - q0) & ~7)) * 2u;
        } else {
            vq[i] = (uint32_t)(min(c >> 3, a.qn - 1 - q0) * (int)a.ldq[0] + 8 * ((c & 7) ^ swz_q(c >> 3))) * 2u;
        }
    }
    // a step's chunks of P and Q straight into LDS; TAIL: zeros past the last k
    auto load = [&](auto tail, int step, int buf) {
        constexpr bool TAIL = decltype(tail)::value;
        const int seg = a.segs > 1 && step >= ksteps ? 1 : 0;
        const int k0 = (step - seg * ksteps) * BK;
        uint8_t *lp = lds[buf] + wave * 1024, *lq = lp + C::PB;
#pragma unroll
        for (int i = 0; i < C::LP; ++i) {
            const int c = i * C::NT + tid;
            const uint8_t *b;
            int k;
            if constexpr (C::PKS) {
                b = (const uint8_t *)a.p[seg] + ((int64_t)k0 * a.ldp[seg] + p0) * 2;
                k = c / (C::TP / 8);
            } else {
                const int mat = KIND == G_GATED ? ((i * C::NT / 8 + wave * 8) >> 5) & 1 : 0;
                b = (const uint8_t *)a.p[mat] + ((int64_t)p0 * a.ldp[mat] + k0) * 2;
                k = 8 * ((c & 7) ^ swz_p<KIND>(c >> 3));
            }
            const uint8_t *src = b + vp[i];
            if (TAIL && k0 + k >= a.kn) src = (const uint8_t *)a.zeros;
            __builtin_amdgcn_global_load_lds(GLB_PTR(src), LDS_PTR(lp + i * C::NT * 16), 16, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < C::LQ; ++i) {
            const int c = i * C::NT + tid;
            const uint8_t *b;
            int k;
            if constexpr (C::QKS) {
                b = (const uint8_t *)a.q[z] + ((int64_t)k0 * a.ldq[z] + q0) * 2;
                k = c / (C::TQ / 8);
            } else {
                b = (const uint8_t *)a.q[seg] + ((int64_t)q0 * a.ldq[seg] + k0) * 2;
                k = 8 * ((c & 7) ^ swz_q(c >> 3));
            }
            const uint8_t *src = b + vq[i];
            if (TAIL && k0 + k >= a.kn) src = (const uint8_t *)a.zeros;
            __builtin_amdgcn_global_load_lds(GLB_PTR(src), LDS_PTR(lq + i * C::NT * 16), 16, 0, 0);
        }
    };
    const bool ragged = a.kn % BK != 0;
    auto fetch = [&](int step, int buf) {
        if (ragged && (step == ksteps - 1 || step == 2 * ksteps - 1)) load(std::true_type{}, step, buf);
        else load(std::false_type{}, step, buf);
    };

    f4_t acc[MT][4];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[m][j] = f4_t{0.f, 0.f, 0.f, 0.f};

    auto tr = [&](const uint8_t *p) {
        return __builtin_bit_cast(V4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4_t *)p));
    };
    auto across = [&](const uint8_t *base, int tcols, int swz, int s, int unit) {
        const int k = 32 * s + 8 * g + (r >> 2);
        const uint8_t *p = base + k * tcols * 2 + (((unit << 1) ^ swz) + ((r >> 1) & 1)) * 16 + (r & 1) * 8;
        const V4 lo = tr(p), hi = tr(p + 4 * tcols * 2);
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    V8 fp[2][4], fq[2][MT];
    auto fragments = [&](int buf, int s) {
        const uint8_t *lp = lds[buf], *lq = lds[buf] + C::PB;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (C::PKS) fp[s][j] = across(lp, C::TP, swz_k<C::TP>(8 * g + (r >> 2)), s, 4 * wp + j);
            else {
                const int row = KIND == G_GATED ? 64 * wp + 32 * (j >> 1) + 8 * (r >> 2) + 4 * (j & 1) + (r & 3)
                                                : 64 * wp + 16 * (r >> 2) + 4 * j + (r & 3);
                fp[s][j] = *(const V8 *)(lp + row * 128 + ((4 * s + g) ^ swz_p<KIND>(row)) * 16);
            }
        }
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            if constexpr (C::QKS) fq[s][m] = across(lq, C::TQ, swz_k<C::TQ>(8 * g + (r >> 2)), s, MT * wq + m);
            else {
                const int row = 16 * (MT * wq + m) + r;
                fq[s][m] = *(const V8 *)(lq + row * 128 + ((4 * s + g) ^ swz_q(row)) * 16);
            }
        }
    };
    // one half of a step, its products spread between the reads of the next half
    auto multiply = [&](int s) {
        constexpr int READS = (C::PKS ? 8 : 4) + (C::QKS ? 2 : 1) * MT, MMAS = 4 * MT, EACH = MMAS / READS;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[m][j] = X::mma(fp[s][j], fq[s][m], acc[m][j]);
        if constexpr (!C::PKS) {
#pragma unroll
        for (int i = 0; i < READS; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);  // an LDS read
            __builtin_amdgcn_sched_group_barrier(0x8, EACH, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x8, MMAS - READS * EACH, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    };

    // At most `steps` steps of loads are still on their way, and every wave's
    // part of the others has arrived.
    auto arrived = [&](auto steps) {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(decltype(steps)::value * (C::LP + C::LQ)) : "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    if (s0 < s1) {
#pragma unroll
        for (int i = 0; i < NS; ++i)
            if (s0 + i < s1) fetch(s0 + i, i);
        if (s0 + NS <= s1) arrived(std::integral_constant<int, NS - 1>{});
        else arrived(std::integral_constant<int, 0>{});
        fragments(0, 0);
        int buf = 0;
        for (int t = s0; t < s1; ++t) {
            const int next = buf + 1 < NS ? buf + 1 : 0;
            fragments(buf, 1);
            multiply(0);
            // the next step has arrived, and every wave has read this one
            if (NS > 2 && t + NS - 1 < s1) arrived(std::integral_constant<int, NS - 2>{});
            else arrived(std::integral_constant<int, 0>{});
            if (t + NS < s1) fetch(t + NS, buf);
            __builtin_amdgcn_s_setprio(1);
            fragments(next, 0);  // (after the last step: not used)
            multiply(1);
            __builtin_amdgcn_s_setprio(0);
            buf = next;
        }
    }
    if (u.tile >= 0) leave_part<C::NT, MT>(a, u, acc);
    else epilogue<X, KIND, MT>(a, acc, q0 + 16 * MT * wq, p0 + (KIND == G_GATED ? 32 : 64) * wp, z);
}

// NS: stages in LDS, or 0: through registers, PF steps ahead.
template <class X, int KIND, int NWQ, int NWP, int MT, int NS, int PF = 1>
static hipError_t launch_tile(const LayerWork &w, GemmArgs a, hipStream_t s)
{
    using C = Tile<X, KIND, NWQ, NWP, MT>;
    double steps;
    if (!lay_out<C, KIND>(w, a, C::per_cu(NS ? NS : 2), &steps)) return hipErrorInvalidConfiguration;
    const int ntile = a.tp * a.tq * a.batch;
    if (ntile == 0) return hipSuccess;
    const hipError_t e = launch_parts(a.full + (ntile - a.full) * a.splits, C::NT, [&](int32_t first, dim3 grid) {
        a.first = first;
        if constexpr (NS != 0) hipLaunchKernelGGL((k_block<X, KIND, NWQ, NWP, MT, NS>), grid, dim3(C::NT), 0, s, a);
        else hipLaunchKernelGGL((k_tile<X, KIND, NWQ, NWP, MT, PF>), grid, dim3(C::NT), 0, s, a);
    });
    if (e != hipSuccess) return e;
    if (a.splits > 1)
        hipLaunchKernelGGL((k_join<X, KIND, NWQ, NWP, MT>), dim3((unsigned)((ntile - a.full) * MT)), dim3(C::NT), 0, s, a);
    return hipGetLastError();
}

// Microseconds that a call takes with each of the tiles: its steps, at what a
// step of each costs with all compute units at it.  bf16 products of 4096 and 8192
// rows, TFLOP/s forward / backward: 256x256 1250 to 1380 / 1160 to 1320; 128x128
// with four stages 790 to 920 / 570 to 640; 64x128 with three, two workgroups to a
// compute unit, 750 to 840 / 650 to 690.  So the backward products, which read
// operands stored across k, have no use for 128x128 (dx of 2048 columns, 320 tokens:
// 19.1 us, 64x128 17.1; 4096x4096, 1024 tokens: 60.4, 56.5, 256x256 53.2).  Over
// forward and backward products of 40 to 4096 tokens and 1024 to 11008 columns the
// choice is 1 to 2% from the best of the tiles, at most 25%.
template <class X, int KIND> static double estimate(const LayerWork &w, GemmArgs a, int tile)
{
    double steps = 0;
    bool ok;
    if (tile == 0) ok = lay_out<Tile<X, KIND, 2, 4, 8>, KIND>(w, a, 1, &steps), steps *= 1.75;
    else if (tile == 1) ok = lay_out<Tile<X, KIND, 4, 2, 2>, KIND>(w, a, 1, &steps), steps *= 0.66;
    else ok = lay_out<Tile<X, KIND, 2, 2, 2>, KIND>(w, a, 2, &steps), steps *= 0.76;
    return ok ? steps : 1e30;
}

template <class X, int KIND> static hipError_t launch_kind(const LayerWork &w, const GemmArgs &a, hipStream_t s)
{
    if (!a.chunks) {
        // (gated 50x4097->5001 bf16: 37 us with 64 rows and two steps ahead, 48 with
        // 128 and one; 100 tokens: 56 and 47)
        if (a.qn <= 64) return launch_tile<X, KIND, 2, 2, 2, 0, 2>(w, a, s);
        return launch_tile<X, KIND, 2, 2, 4, 0, 1>(w, a, s);
    }
    constexpr bool FORWARD = KIND == G_LINEAR || KIND == G_GATED;
    int tile = 0;
    for (int i = FORWARD ? 1 : 2; i < 3; ++i)
        if (estimate<X, KIND>(w, a, i) < estimate<X, KIND>(w, a, tile)) tile = i;
    if (tile == 0) return launch_tile<X, KIND, 2, 4, 8, 2>(w, a, s);
    if constexpr (FORWARD)
        if (tile == 1) return launch_tile<X, KIND, 4, 2, 2, 4>(w, a, s);
    return launch_tile<X, KIND, 2, 2, 2, 3>(w, a, s);
}

template <class X> hipError_t launch_type(const LayerWork &w, GemmKind kind, const GemmArgs &a, hipStream_t s)
{
    switch (kind) {
    case G_LINEAR: return launch_kind<X, G_LINEAR>(w, a, s);
    case G_GATED: return launch_kind<X, G_GATED>(w, a, s);
    case G_DX: return launch_kind<X, G_DX>(w, a, s);
    default: return launch_kind<X, G_DW>(w, a, s);
    }
}

bool whole_chunks(const void *p, int64_t ld, int64_t contiguous)
{
    return (uintptr_t)p % 16 == 0 && ld % 8 == 0 && ld <= (1 << 21) && contiguous % 8 == 0;
}

hipError_t launch_gemm(const LayerWork &w, bool bf16, GemmKind kind, GemmArgs a, hipStream_t s)
{
    a.zeros = w.zeros, a.part = w.part;
    if ((kind == G_LINEAR || kind == G_GATED) && rows_take(kind == G_GATED, a))
        return launch_rows(w, bf16, kind == G_GATED, a, s);
    const bool pks = kind == G_DX || kind == G_DW, qks = kind == G_DW;
    const int np = kind == G_GATED || kind == G_DX ? (kind == G_GATED ? 2 : a.segs) : 1;
    const int nq = kind == G_DX ? a.segs : a.batch;
    a.chunks = 1;
    for (int i = 0; i < np; ++i)
        a.chunks &= whole_chunks(a.p[i], a.ldp[i], a.p_padded ? 0 : pks ? a.pn : a.kn) && (kind != G_DX || a.ldp[i] == a.ldp[0]);
    for (int i = 0; i < nq; ++i)
        a.chunks &= whole_chunks(a.q[i], a.ldq[i], a.q_padded ? 0 : qks ? a.qn : a.kn) && a.ldq[i] == a.ldq[0];
    return bf16 ? launch_type<Bf16>(w, kind, a, s) : launch_type<Fp16>(w, kind, a, s);
}

}  // namespace dbs
