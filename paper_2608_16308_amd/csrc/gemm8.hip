// Products of matrices in blocks of 8-bit floating point on the matrix cores.
#include <algorithm>
#include <utility>

#include "float8.hpp"
#include "layer_tile.hpp"

namespace dbs {

typedef int v8i_t __attribute__((ext_vector_type(8)));
typedef int v4i_t __attribute__((ext_vector_type(4)));

// A step is one block, E8_BLOCK elements of the sum: bytes of a row in LDS as
// BK elements of 16 bits, so the order of a tile in LDS, its place and its epilogue
// are those of the 16-bit products.
static_assert(E8_BLOCK == 2 * BK, "a step is a block");

struct Gemm8Args {
    GemmArgs g;
    const uint8_t *pe, *qe;   // exponents
    int64_t ldpe, ldqe;
    int32_t pshift;
    int32_t steps;            // blocks along k; g.kn counts them in quads of four
};

// One 16x16x128 step: the matrix cores multiply by 2^(sp - 127) and 2^(sq - 127),
// byte SP (SQ) of a lane being the scale of its row's block.
//
// They add eight neighbouring products in fixed point, cut to multiples of 2^(E -
// 13) with 2^E <= the largest of the eight, and the sums of eight in 32 bits; all
// their 8-bit products do.  That is the price of twice the rate of 16 bits: an
// error that is small beside the rounding of the result (1531x7001->5003 in fp16:
// 2.1e-4 from 64 bits in the norm, as the product in 32 bits is).
template <int SP, int SQ> __device__ __forceinline__ f4_t mma8(v8i_t p, v8i_t q, f4_t c, int sp, int sq)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(p, q, c, 0, 0, SP, sp, SQ, sq);
}

__device__ __forceinline__ uint32_t lds_at(void *p) { return (uint32_t)(uintptr_t)LDS_PTR(p); }
// N bytes a lane from base + off straight into LDS, the lanes' behind each other
// from `to` on.  Written as asm because the compiler, which sees such a load as a
// write to all of LDS, waits for every one on its way before it reads anything
// there; the kernel's own waits are counted instead.  (It returns no register, so
// nothing can be taken for written too soon; m0, the place, is named as written, so that
// no use of it by the compiler is taken to outlast this, and the warning that the
// compiler reserves it says no more than that.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
template <int N> __device__ __forceinline__ void to_lds(const uint8_t *base, uint32_t off, uint32_t to)
{
    if constexpr (N == 16) asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(base) : "m0");
    else asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(to), "v"(off), "s"(base) : "m0");
}
#pragma clang diagnostic pop

// f(0), f(1) .. f(N - 1) with the number known to the compiler.
template <class F, int... I> __device__ __forceinline__ void each_of(F &&f, std::integer_sequence<int, I...>)
{
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F> __device__ __forceinline__ void each(F &&f) { each_of(f, std::make_integer_sequence<int, N>{}); }

// Rounds and stores a wave's 16 MT x 64 sums, a lane's columns 16 in a row.
template <class X, int MT>
__device__ __forceinline__ void finish(const GemmArgs &a, const f4_t (&acc)[MT][4], int q0, int p0)
{
    typedef typename X::T T;
    typedef typename X::V8 V8;
    const int lane = lane_id(), col = p0 + 16 * (lane >> 4), left = a.pn - col;
    if (left <= 0) return;
    V8 bias[2] = {};
    if (a.bias) {
        const T *b = (const T *)a.bias + col;
        if (left >= 16) bias[0] = load_eight<X>(b), bias[1] = load_eight<X>(b + 8);
        else
#pragma unroll
            for (int i = 0; i < 16; ++i) bias[i >> 3][i & 7] = i < left ? b[i] : (T)0.f;
    }
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int row = q0 + 16 * m + (lane & 15);
        if (row >= a.qn) continue;
        T *dst = (T *)a.y[0] + (int64_t)row * a.ldy[0] + col;
        const T *res = a.res ? (const T *)a.res + (int64_t)row * a.ldr + col : nullptr;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            V8 o, add = {};
            if (left >= 16) {
                if (res) add = load_eight<X>(res + 8 * h);
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i] = (T)(acc[m][2 * h + (i >> 2)][i & 3] + (float)bias[h][i] + (float)add[i]);
                store_any(dst + 8 * h, o);
            } else
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (8 * h + i < left)
                        dst[8 * h + i] = (T)(acc[m][2 * h + (i >> 2)][i & 3] + (float)bias[h][i] + (res ? (float)res[8 * h + i] : 0.f));
        }
    }
}

// Sizes of a tile: four waves, each with 16 MT rows of q and 64 H of p; NS steps in
// LDS; fragments of q are read PD rows of products ahead.
template <int MT, int H, int NS> struct Tile8 {
    static constexpr int NT = 256, TQ = 32 * MT, TP = 128 * H;
    static constexpr int PB = TP * E8_BLOCK, QB = TQ * E8_BLOCK;
    static constexpr int LP = PB / 16 / NT, LQ = QB / 16 / NT;  // chunks per thread and step
    static constexpr int ROWS = TP + TQ, NW = (ROWS + NT - 1) / NT;  // rows with exponents; per thread
    static constexpr int PD = MT >= 8 ? 3 : MT / 2, RING = MT >= 8 ? 4 : MT;
    static constexpr int LDS = NS * (PB + QB) + 12 * ROWS + 256;
    static constexpr int PER_CU = 160 * 1024 / LDS;
};

// A tile of the product, chunks straight into LDS.  Four waves of up to 128x128
// products each read half as much of LDS for a product as eight of 128x64 would,
// which the 16-bit tiles can afford, and these not: their products take half the
// time.  With one wave to a SIMD nothing else hides its waits, so the code does:
// while a row of products (16 rows of q) runs, the fragments of a later one are
// read, and from the row on at which all of this step's have been, those of the
// next step, whose arrival all waves have waited for at the one barrier of a step.
//
// Exponents come four steps at a time (a quad), a word for each row, through
// registers into an order in LDS that gives a lane all of a step's in one read.
//
// Bound by the waits for lines that are not in L2 (with all of them there a fifth of the
// time is gone; the matrix cores are busy 49% of it): 8192x8192->8192 in bf16 436 us,
// 2520 TFLOP/s; 4096x11008->4096 142 (2600), 4096x4096->11008 177 (2090: 2.7 rounds of
// tiles).
template <class X, int MT, int H, int NS>
__global__ __launch_bounds__(256, (Tile8<MT, H, NS>::PER_CU)) void k_mul8(Gemm8Args b)
{
    using C = Tile8<MT, H, NS>;
    const GemmArgs &a = b.g;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[NS][C::PB + C::QB];
    __shared__ __attribute__((aligned(16))) uint8_t exps[2][4][C::ROWS];
    __shared__ uint32_t words[C::ROWS];
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = wave_id();
    const int wq = wave >> 1, wp = wave & 1, r = lane & 15, g = lane >> 4;
    const Unit u = unit_of<C::TQ, C::TP>(a);
    const int q0 = u.q0, p0 = u.p0, s0 = 4 * u.s0, s1 = min(4 * u.s1, b.steps);

    // A thread's chunks are 32 rows apart; `v` is the place of one within its 32 rows.
    // Of an operand's last tile the rows past the end are read as the last one (`end`),
    // groups of 32 without any row as the last group.
    const int row = tid >> 3;
    const int rows_p = min(a.pn - p0, C::TP), rows_q = min(a.qn - q0, C::TQ);  // rows there
    const uint32_t ldp = (uint32_t)a.ldp[0], ldq = (uint32_t)a.ldq[0];
    const uint32_t vp = row * ldp + 16u * ((tid & 7) ^ swz_p<G_LINEAR>(row)), vq = row * ldq + 16u * ((tid & 7) ^ swz_q(row));
    const uint32_t end_p = vp - (uint32_t)max(row - (rows_p - 1) % 32, 0) * ldp, end_q = vq - (uint32_t)max(row - (rows_q - 1) % 32, 0) * ldq;
    const uint8_t *bp = (const uint8_t *)a.p[0] + (int64_t)p0 * a.ldp[0], *bq = (const uint8_t *)a.q[0] + (int64_t)q0 * a.ldq[0];
    // chunk i of a thread, of step `step` (P's before Q's)
    auto fetch = [&](int step, int buf, auto ic) {
        constexpr int I = decltype(ic)::value;
        const uint32_t to = lds_at(lds[buf]) + I * C::NT * 16 + wave * 1024;
        constexpr int G = I < C::LP ? I : I - C::LP;
        const int last = ((I < C::LP ? rows_p : rows_q) - 1) / 32, group = min(G, last);
        if constexpr (I < C::LP) to_lds<16>(bp + (int64_t)step * E8_BLOCK + group * 32u * ldp, G < last ? vp : end_p, to);
        else to_lds<16>(bq + (int64_t)step * E8_BLOCK + group * 32u * ldq, G < last ? vq : end_q, to);
    };
    // The workgroups of an XCD that run beside each other share their rows of P by four
    // (those of a group of tiles) and of Q by eight: each asks for its share of a later
    // step's lines once, so that the loads of all find them in L2.  What is read is not
    // used.  (The large tile has two stages, one step of time for a load: 4096x4096 ->
    // 11008 190 -> 182 us, 8192^3 469 -> 436.  The others, with more, lose 2% by it.)
    constexpr bool ASK = NS == 2;
    __shared__ uint32_t asked[ASK ? 64 : 1];
    auto ask = [&](int step) {
        const int q = q0 / C::TQ & 3, p = p0 / C::TP & 7, n = wave < 2 ? C::TP / 8 : C::TQ / 16;
        const int first = wave < 2 ? q * (C::TP / 4) + wave * n : p * (C::TQ / 8) + (wave - 2) * n;
        int l = lane;
        asm volatile("" : "+v"(l));  // (registers are short: worked out again each time)
        if (l < n)
            to_lds<4>((wave < 2 ? bp : bq) + (int64_t)step * E8_BLOCK, (uint32_t)min(first + l, (wave < 2 ? rows_p : rows_q) - 1) * (wave < 2 ? ldp : ldq),
                      lds_at(asked));
    };
    // the exponents of a thread's rows, and their place (worked out again each time:
    // registers are short)
    auto rows_of = [&](int i, auto &&of) {
        int e = tid;
        asm volatile("" : "+v"(e));
        e += i * C::NT;
        if ((i + 1) * C::NT > C::ROWS && i * C::NT + wave * 64 >= C::ROWS) return;
        if (i * C::NT + wave * 64 < C::TP) {  // (the same for all lanes of a wave: tiles have whole waves of rows)
            const int64_t first = (int64_t)(p0 >> b.pshift) * b.ldpe;
            of(b.pe + first, (uint32_t)(((int64_t)min(p0 + e, a.pn - 1) >> b.pshift) * b.ldpe - first),
               (e & -64 * H) + (((e >> 4) & 3) * 4 + (e & 3)) * 4 * H + (H > 1 ? (e >> 4) & 4 : 0) + ((e >> 2) & 3));
        } else {
            const int q = e - C::TP;
            of(b.qe + q0 * b.ldqe, (uint32_t)(min(q, a.qn - 1 - q0) * b.ldqe),
               C::TP + q / (16 * MT) * (16 * MT) + (q & 15) * MT + (q >> 4) % MT);
        }
    };
    auto load_words = [&](int quad) {
#pragma unroll
        for (int i = 0; i < C::NW; ++i)
            rows_of(i, [&](const uint8_t *base, uint32_t off, int) { to_lds<4>(base + 4 * quad, off, lds_at(words) + 4 * (i * C::NT + wave * 64)); });
    };
    auto put_words = [&](int half) {
#pragma unroll
        for (int i = 0; i < C::NW; ++i)
            rows_of(i, [&](const uint8_t *, uint32_t, int at) {
                const uint32_t w = words[i * C::NT + tid];
#pragma unroll
                for (int s = 0; s < 4; ++s) exps[half][s][at] = (uint8_t)(w >> (8 * s));
            });
    };

    f4_t acc[H][MT][4];
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[h][m][j] = f4_t{0.f, 0.f, 0.f, 0.f};

    // a lane's 32 elements of a row (in the same order for p and q; the sum does
    // not depend on it, since a block has one scale)
    auto fragment = [&](const uint8_t *tile, int row, int swz) {
        const v4i_t lo = *(const v4i_t *)(tile + row * E8_BLOCK + (g ^ swz) * 16), hi = *(const v4i_t *)(tile + row * E8_BLOCK + ((4 + g) ^ swz) * 16);
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    v8i_t fp[2][4 * H], fq[C::RING];
    int ep[2][H], eq[2][MT >= 8 ? 2 : 1];
    auto read_p = [&](int buf, int set, int i) {
        const int row = 64 * H * wp + 64 * (i >> 2) + 16 * (r >> 2) + 4 * (i & 3) + (r & 3);
        fp[set][i] = fragment(lds[buf], row, swz_p<G_LINEAR>(row));
    };
    auto read_q = [&](int buf, int m) {
        const int row = 16 * (MT * wq + m) + r;
        fq[m % C::RING] = fragment(lds[buf] + C::PB, row, swz_q(row));
    };
    auto read_exps = [&](int half, int s, int set) {
        const uint8_t *e = exps[half][s], *p = e + 64 * H * wp + 4 * H * r, *q = e + C::TP + 16 * MT * wq + MT * r;
#pragma unroll
        for (int h = 0; h < H; ++h) ep[set][h] = *(const int *)(p + 4 * h);
        if constexpr (MT == 2) eq[set][0] = *(const uint16_t *)q;
        else
#pragma unroll
            for (int i = 0; i < MT / 4; ++i) eq[set][i] = *(const int *)(q + 4 * i);
    };
    // At most `loads` loads are still on their way, and every wave's part of the
    // others has arrived.
    auto arrived = [&](auto loads) {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(decltype(loads)::value) : "memory");
        __builtin_amdgcn_sched_barrier(0);
    };

    if (s0 < s1) {
        load_words(u.s0);
        each<NS>([&](auto n) {
            each<C::LP + C::LQ>([&](auto i) { fetch(min(s0 + decltype(n)::value, s1 - 1), decltype(n)::value, i); });
        });
        arrived(std::integral_constant<int, (NS - 1) * (C::LP + C::LQ)>{});
        put_words(0);
        __syncthreads();
        read_exps(0, 0, 0);
        each<4 * H>([&](auto i) { read_p(0, 0, i); });
        each<C::PD>([&](auto m) { read_q(0, m); });
        int buf = 0;
        for (int quad = u.s0; 4 * quad < s1; ++quad) {
            const int half = (quad - u.s0) & 1;
            each<4>([&](auto sc) {
                constexpr int S = decltype(sc)::value, SET = S & 1;
                const int t = 4 * quad + S;
                if (t >= s1) return;
                const int next = buf + 1 < NS ? buf + 1 : 0;
                each<MT>([&](auto mc) {
                    constexpr int M = decltype(mc)::value, FREE = MT - C::PD;  // the row at which all of a step has been read
                    if constexpr (M == FREE) {
                        // the next step has arrived, and every wave has read this one
                        arrived(std::integral_constant<int, (NS - 2) * (C::LP + C::LQ) + ASK>{});
                        if (S == 2) put_words(half ^ 1);
                        if (S == 0) load_words(min(quad + 1, u.s1 - 1));
                        read_exps(S == 3 ? half ^ 1 : half, (S + 1) & 3, SET ^ 1);
                    }
                    if constexpr (ASK && M == 0) ask(min(t + 3, s1 - 1));  // (the last load of all that the wait counts)
                    if constexpr (M < FREE) read_q(buf, M + C::PD);
                    else {
                        // (behind the last step: the last one again, read and not used, so that
                        // the waits count the same loads in every step)
                        read_q(next, M - FREE);
                        constexpr int FROM = (M - FREE) * 4 * H / C::PD, TO = (M - FREE + 1) * 4 * H / C::PD;
                        each<TO - FROM>([&](auto i) { read_p(next, SET ^ 1, FROM + decltype(i)::value); });
                        constexpr int LF = (M - FREE) * (C::LP + C::LQ) / C::PD, LT = (M - FREE + 1) * (C::LP + C::LQ) / C::PD;
                        each<LT - LF>([&](auto i) { fetch(min(t + NS, s1 - 1), buf, std::integral_constant<int, LF + decltype(i)::value>{}); });
                    }
                    each<H>([&](auto hc) {
                        constexpr int HH = decltype(hc)::value;
                        each<4>([&](auto jc) {
                            constexpr int J = decltype(jc)::value;
                            acc[HH][M][J] = mma8<J, (M & 3)>(fp[SET][4 * HH + J], fq[M % C::RING], acc[HH][M][J], ep[SET][HH], eq[SET][M >> 2]);
                        });
                    });
                });
                buf = next;
            });
        }
        arrived(std::integral_constant<int, 0>{});
    }
    if (u.tile >= 0) {
        // (in the order in which k_join has a tile of 2 x 2 H waves)
        constexpr int NV = 256 * H;
#pragma unroll
        for (int h = 0; h < H; ++h) {
            f4_t *own = (f4_t *)a.part + (int64_t)(u.tile * a.splits + u.part) * MT * 4 * NV + (2 * H * wq + H * wp + h) * 64 + lane;
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int j = 0; j < 4; ++j) own[(m * 4 + j) * NV] = acc[h][m][j];
        }
    } else
        each<H>([&](auto h) { finish<X, MT>(a, acc[decltype(h)::value], q0 + 16 * MT * wq, p0 + 64 * (H * wp + decltype(h)::value)); });
}

// The tiles of a call, how many of them are taken whole and in how many parts the
// others; microseconds that this takes, a quad with all compute units at it taking
// `quad` (`alone` with one tile on each), and joining a launch and the bytes of the
// parts written and read.
template <class C> static double lay_out8(const LayerWork &w, GemmArgs &a, double quad, double alone)
{
    const int64_t tq = ((int64_t)a.qn + C::TQ - 1) / C::TQ, tp = ((int64_t)a.pn + C::TP - 1) / C::TP, ntile = tq * tp;
    if (ntile > MAX_TILES) return 1e30;
    a.tq = (int32_t)tq, a.tp = (int32_t)tp;
    const int64_t slots = (int64_t)w.cus * C::PER_CU, quads = a.kn / BK, rest = ntile % slots;
    a.full = (int32_t)(ntile - rest), a.splits = 1;
    const double whole = (double)(ntile / slots) * (double)quads * quad;
    if (rest == 0) return whole;
    auto round = [&](int64_t parts) { return parts <= w.cus ? alone : quad; };
    double best = (double)quads * round(rest);
    for (int64_t s = 2; s <= 16 && s <= quads; ++s) {
        const int64_t bytes = rest * s * C::TP * C::TQ * 4;
        if (bytes > (int64_t)w.part_bytes) break;
        const double cost = (double)((rest * s + slots - 1) / slots) * (double)((quads + s - 1) / s) * round(rest * s) + 4 + (double)bytes * 0.45e-6;
        if (cost < best) best = cost, a.splits = (int32_t)s;
    }
    return whole + best;
}

template <class X, int MT, int H, int NS> static hipError_t launch_tile8(const LayerWork &w, Gemm8Args b, double quad, double alone, hipStream_t s)
{
    using C = Tile8<MT, H, NS>;
    if (lay_out8<C>(w, b.g, quad, alone) >= 1e30) return hipErrorInvalidConfiguration;
    const int ntile = b.g.tp * b.g.tq;
    const hipError_t e = launch_parts(b.g.full + (int64_t)(ntile - b.g.full) * b.g.splits, C::NT, [&](int32_t first, dim3 grid) {
        b.g.first = first;
        hipLaunchKernelGGL((k_mul8<X, MT, H, NS>), grid, dim3(C::NT), 0, s, b);
    });
    if (e != hipSuccess) return e;
    if (b.g.splits > 1)
        hipLaunchKernelGGL((k_join<X, G_LINEAR, 2, 2 * H, MT>), dim3((unsigned)((ntile - b.g.full) * MT)), dim3(256 * H), 0, s, b.g);
    return hipGetLastError();
}

// Which tile: the one with the least time by the rule above.  us with each tile forced
// (256x256, 128x128, 128x256 and 64x128 of q and p), bf16, both factors in blocks, calls back to
// back, so that the last-level cache has the factors (1531x7001->5003 in fp16 56 us so, 70
// behind the packing of x in a call of its own; the rule has not been measured there):
//   17x4096->4096         31.9    16.3    22.0    13.9
//   256x4096->11008       35.4    23.0    28.3    23.6
//   512x4096->4096        30.1    21.9    25.0    17.0
//   777x11008->4096       59.2    47.4    51.1    57.7
//   777x4096->11008       61.9    60.9    54.5    54.5
//   1531x7001->5003       69.4    65.6    56.2    71.3
//   2048x4096->11008     104.4   118.1   101.0   114.4
//   4096x4096->4096       61.8    80.1    70.7    84.4
//   4096x4096->11008     176.8   217.4   202.1   229.6
// (a tile that has a compute unit for itself takes a quad in 1.65 us, two in 2.53: without
// the difference 512x4096->4096 went to 128x128, 64x4096->11008 to fewer parts, 17.6 us for 15.3)
template <class X> static hipError_t mul8_t(const LayerWork &w, const Gemm8Args &b, hipStream_t s)
{
    constexpr double BIG = 6.75, SQUARE = 2.25, FLAT = 3.8, SMALL = 2.53, SMALL_ALONE = 1.65;
    GemmArgs g = b.g;
    const double big = lay_out8<Tile8<8, 2, 2>>(w, g, BIG, BIG), square = lay_out8<Tile8<4, 1, 4>>(w, g, SQUARE, SQUARE);
    const double flat = lay_out8<Tile8<4, 2, 3>>(w, g, FLAT, FLAT), small = lay_out8<Tile8<2, 1, 3>>(w, g, SMALL, SMALL_ALONE);
    const double least = std::min(std::min(big, square), std::min(flat, small));
    if (least == big) return launch_tile8<X, 8, 2, 2>(w, b, BIG, BIG, s);
    if (least == square) return launch_tile8<X, 4, 1, 4>(w, b, SQUARE, SQUARE, s);
    if (least == flat) return launch_tile8<X, 4, 2, 3>(w, b, FLAT, FLAT, s);
    return launch_tile8<X, 2, 1, 3>(w, b, SMALL, SMALL_ALONE, s);
}

hipError_t launch_mul8(const LayerWork &w, bool bf16, const Mul8Args &m, hipStream_t s)
{
    if (m.pn == 0 || m.qn == 0) return hipSuccess;
    Gemm8Args b{};
    b.g.p[0] = m.p.codes, b.g.ldp[0] = m.p.ld, b.g.q[0] = m.q.codes, b.g.ldq[0] = m.q.ld;
    b.g.pn = m.pn, b.g.qn = m.qn, b.g.kn = (int32_t)((e8_blocks(m.kn) + 3) / 4 * BK), b.g.segs = 1, b.g.batch = 1;
    b.g.y[0] = m.y, b.g.ldy[0] = m.ldy, b.g.bias = m.bias, b.g.res = m.res, b.g.ldr = m.ldr, b.g.act = Act::of(DBS_ACT_NONE);
    b.g.part = w.part;
    b.steps = (int32_t)e8_blocks(m.kn);
    b.pe = m.p.exps, b.ldpe = m.p.lde, b.pshift = m.p.shift, b.qe = m.q.exps, b.ldqe = m.q.lde;
    return bf16 ? mul8_t<Bf16>(w, b, s) : mul8_t<Fp16>(w, b, s);
}

}  // namespace dbs
