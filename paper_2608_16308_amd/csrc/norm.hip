// Norms before and after a block, the join with the residual stream, dropout,
// and their gradients.
#include <algorithm>
#include <type_traits>

#include "float8.hpp"
#include "norm.hpp"

namespace dbs {

// Eight elements in words; `left` of them (1 to 7), at any alignment, as four, two
// and one.
struct Words {
    uint32_t w[4];
};
struct __attribute__((packed, aligned(2))) Four {
    uint32_t w[2];
};
struct __attribute__((packed, aligned(2))) Two {
    uint32_t w;
};
__device__ __forceinline__ Words get_part(const void *p, int left)
{
    const uint16_t *at = (const uint16_t *)p;
    Words r = {{0u, 0u, 0u, 0u}};
    uint32_t lo = 0, hi = 0;  // what follows the four
    if (left & 1) lo = at[left & 6];
    if (left & 2) {
        const uint32_t two = ((const Two *)(at + (left & 4)))->w;
        hi = lo, lo = two;
    }
    if (left & 4) {
        const Four four = *(const Four *)at;
        r.w[0] = four.w[0], r.w[1] = four.w[1], r.w[2] = lo, r.w[3] = hi;
    } else r.w[0] = lo, r.w[1] = hi;
    return r;
}
__device__ __forceinline__ void put_part(void *p, int left, Words v)
{
    uint16_t *at = (uint16_t *)p;
    if (left & 4) {
        *(Four *)at = Four{{v.w[0], v.w[1]}};
        v.w[0] = v.w[2], v.w[1] = v.w[3];
    }
    if (left & 2) {
        ((Two *)(at + (left & 4)))->w = v.w[0];
        v.w[0] = v.w[1];
    }
    if (left & 1) at[left & 6] = (uint16_t)v.w[0];
}
template <class X> __device__ __forceinline__ void put_eight(typename X::T *p, int left, const float (&v)[8])
{
    typename X::V8 t;
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = (typename X::T)v[i];
    if (left >= 8) ((Eight<X> *)p)->v = t;
    else if (left > 0) put_part(p, left, __builtin_bit_cast(Words, t));
}
// Eight elements of a row of which `left` are there; the rest reads as zeros.
template <class X> __device__ __forceinline__ typename X::V8 get_eight(const typename X::T *p, int left)
{
    typename X::V8 v = {};
    if (left >= 8) v = load_eight<X>(p);
    else if (left > 0) v = __builtin_bit_cast(typename X::V8, get_part(p, left));
    return v;
}
template <class X> __device__ __forceinline__ void get_floats(const typename X::T *p, int left, float (&v)[8])
{
    const typename X::V8 t = get_eight<X>(p, left);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)t[i];
}
// The same of a vector that may be missing: `none` then.
template <class X>
__device__ __forceinline__ typename X::V8 get_vector(const void *p, int col, int left, float none)
{
    if (p) return get_eight<X>((const typename X::T *)p + col, left);
    typename X::V8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (typename X::T)none;
    return v;
}

// Sums over a workgroup, the same in all its threads: `red` holds two rounds, so
// that one barrier each is enough.
template <int WAVES> struct GroupSum {
    float (*red)[WAVES];
    int round = 0;
    __device__ float operator()(float v)
    {
        v = wave_sum(v);
        if (WAVES == 1) return v;
        if (lane_id() == 0) red[round][wave_id()] = v;
        __syncthreads();
        float s = red[round][0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) s += red[round][w];
        round ^= 1;
        return s;
    }
};

// Chunk c of a row of h into 8 bits, the 16 of a block in neighbouring lanes (all
// lanes of the wave come here); `last` chunks make whole blocks.
template <class X>
__device__ __forceinline__ void put_codes(const EdgeArgs &a, int64_t row, int c, int last, const float (&h)[8])
{
    float v[8], big = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)(typename X::T)h[i], big = fmaxf(big, ck_mag(v[i]));
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) big = fmaxf(big, __shfl_xor(big, o, 64));
    if (c >= last) return;
    const int e = e8_exp(big);
    *(uint2 *)(a.codes + row * e8_ld(a.n) + 8 * c) = e8_codes(v, e);
    if (c % 16) return;
    uint8_t *exps = a.exps + row * e8_ldexp(a.n);
    exps[c / 16] = (uint8_t)(e + E8_BIAS);
    if (c + 16 == last)
        for (int b = last / 16; b < (int)e8_ldexp(a.n); ++b) exps[b] = E8_BIAS;
}

__device__ __forceinline__ void rng_of(const Drop &d, uint64_t &seed, uint64_t &offset)
{
    seed = d.rng ? d.rng[0] : d.seed;
    offset = d.rng ? d.rng[1] : d.offset;
}

// What a row is multiplied by where its squares would leave the range of 32 bits (else
// 1), from its variance and mean as it is.  Above 2^128 squares are infinite.  Below 2^-126 they
// lose bits, which counts where variance and eps are below 2^-120: then all of x - mean is
// below 2^-45 (in rows of 2^30), and a mean below 2^20 leaves x 2^100 in range.  (Beside a
// larger mean numbers of 24 bits that differ at all have a larger variance.)
constexpr float DOWN = 8.271806125530277e-25f, UP = 1.2676506002282294e30f;  // 2^-80, 2^100
constexpr float LEAST_VAR = 7.5231638452626401e-37f;                          // 2^-120
__device__ __forceinline__ float again_by(float var, float eps, float mean)
{
    if (var > 3.402823466e38f) return DOWN;
    return var + eps < LEAST_VAR && __builtin_fabsf(mean) < 1048576.f ? UP : 1.f;
}

// The statistics of a row whose values `at(chunk, v)` gives: the mean first, then
// the squares around it, so that a large mean costs no precision.  Eight terms are added
// in 32 bits and these sums in 64: one after the other in 32 bits a lane's 2^18 of a row of 2^28
// equal numbers were off by 0.4%.
template <int WAVES, class F>
__device__ __forceinline__ Stat row_stat(const NormOf &nm, int n, GroupSum<WAVES> &total, F &&at)
{
    const float by = 1.f / (float)n;
    for (float f = 1.f;;) {
        float mean = 0.f;
        double sum = 0.0;
        if (nm.kind == DBS_NORM_LAYER) {
            for (int c = (int)threadIdx.x; 8 * c < n; c += 64 * WAVES) {
                float v[8];
                at(c, v);
                float part = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) part += 8 * c + i < n ? v[i] * f * by : 0.f;
                sum += part;
            }
            mean = total((float)sum), sum = 0.0;
        }
        for (int c = (int)threadIdx.x; 8 * c < n; c += 64 * WAVES) {
            float v[8];
            at(c, v);
            float part = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = 8 * c + i < n ? __builtin_fmaf(v[i], f, -mean) : 0.f;
                part = __builtin_fmaf(d, d, part);
            }
            sum += part;
        }
        const float var = total((float)sum) * by;
        const float again = f == 1.f ? again_by(var, nm.eps, mean) : 1.f;
        if (again == 1.f) return Stat{f, mean, rsqrtf(var + nm.eps * f * f)};
        f = again;
    }
}

// ---------------------------------------------------------------------------
// rows of any length: read again from the caches for each step
// ---------------------------------------------------------------------------
constexpr int LONG_WAVES = 16;

template <class X, bool BRANCH> __global__ __launch_bounds__(64 * LONG_WAVES) void k_edge_long(EdgeArgs a)
{
    typedef typename X::T T;
    __shared__ float red[2][LONG_WAVES];
    GroupSum<LONG_WAVES> total{red};
    uint64_t seed, offset;
    rng_of(a.drop, seed, offset);
    const int64_t chunks = (a.n + 7) / 8;
    for (int row = (int)blockIdx.x; row < a.rows; row += (int)gridDim.x) {
        const T *res = (const T *)a.res + row * a.ldr, *branch = (const T *)a.branch + row * a.ldb;
        Stat sa{};
        if (BRANCH && a.after.kind != DBS_NORM_NONE)
            sa = row_stat(a.after, a.n, total, [&](int c, float(&v)[8]) { get_floats<X>(branch + 8 * c, a.n - 8 * c, v); });
        // the stream, 8 columns of it
        auto stream = [&](int c, float(&s)[8]) {
            const int col = 8 * c, left = a.n - col;
            get_floats<X>(res + col, left, s);
            if constexpr (BRANCH) {
                float u[8];
                get_floats<X>(branch + col, left, u);
                if (a.after.kind != DBS_NORM_NONE) {
                    const typename X::V8 w = get_vector<X>(a.after.w, col, left, 1.f), b = get_vector<X>(a.after.b, col, left, 0.f);
#pragma unroll
                    for (int i = 0; i < 8; ++i) u[i] = __builtin_fmaf(sa.xh(u[i]), (float)w[i], (float)b[i]);
                }
                if (a.drop.threshold) drop_eight(a.drop, seed, offset, row * chunks + c, u);
                const typename X::V8 g = get_vector<X>(a.gate ? (const T *)a.gate + row * a.ldg : nullptr, col, left, 1.f);
#pragma unroll
                for (int i = 0; i < 8; ++i) s[i] = __builtin_fmaf((float)g[i], u[i], a.scale * s[i]);
            }
        };
        Stat sb{};
        if (a.before.kind != DBS_NORM_NONE) sb = row_stat(a.before, a.n, total, stream);
        __syncthreads();  // (the stream may replace the residual)
        const int last = a.codes ? (int)e8_blocks(a.n) * 16 : (int)chunks;
        for (int c = (int)threadIdx.x; c < (last + 63) / 64 * 64; c += 64 * LONG_WAVES) {
            const int col = 8 * c, left = a.n - col;
            float s[8] = {}, h[8] = {};
            if (left > 0) {
                stream(c, s);
                if (BRANCH) put_eight<X>((T *)a.stream + row * a.lds + col, left, s);
                if (a.before.kind != DBS_NORM_NONE) {
                    const typename X::V8 w = get_vector<X>(a.before.w, col, left, 1.f), b = get_vector<X>(a.before.b, col, left, 0.f);
#pragma unroll
                    for (int i = 0; i < 8; ++i) h[i] = i < left ? __builtin_fmaf(sb.xh(s[i]), (float)w[i], (float)b[i]) : 0.f;
                    if (a.h) put_eight<X>((T *)a.h + row * a.ldh + col, left, h);
                }
            }
            if (a.codes) put_codes<X>(a, row, c, last, h);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------
// rows that a workgroup's registers hold
// ---------------------------------------------------------------------------
// The sum over 16 neighbouring lanes, in all of them.
__device__ __forceinline__ float sum16(float v)
{
    auto ror = [](auto ctrl, float x) { return __builtin_bit_cast(float, dpp_mov<decltype(ctrl)::value>(0u, __builtin_bit_cast(uint32_t, x))); };
    v += ror(std::integral_constant<int, dppc::ROW_ROR + 1>{}, v);
    v += ror(std::integral_constant<int, dppc::ROW_ROR + 2>{}, v);
    v += ror(std::integral_constant<int, dppc::ROW_ROR + 4>{}, v);
    v += ror(std::integral_constant<int, dppc::ROW_ROR + 8>{}, v);
    return v;
}
struct Pair {
    float a, b;
};
__device__ __forceinline__ Pair swap16(float x, float y)  // rows x0 y0 x2 y2 and x1 y1 x3 y3
{
    const auto v = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, y), false, false);
    const uint32_t a = v[0], b = v[1];
    return {__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)};
}
__device__ __forceinline__ Pair swap32(float x, float y)  // rows x0 x1 y0 y1 and x2 x3 y2 y3
{
    const auto v = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, y), false, false);
    const uint32_t a = v[0], b = v[1];
    return {__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)};
}
__device__ __forceinline__ float add(Pair v) { return v.a + v.b; }

// A team: the waves that have a row, a workgroup or one of its waves.  Sums over
// it, the same in all its lanes.  One or two values are folded into one register first
// (two: the lower and the upper half of the lanes), so that both take the steps of
// one (join backward of 4096x4096 with two layer norms in fp16 95 -> 91 us).
constexpr int MAX_TEAM = 16;
struct Team {
    float (*red)[2][4][MAX_TEAM];  // [round][register][row of lanes][wave]
    int waves, round;
    template <int N> static __device__ __forceinline__ float fold(const float (&v)[N])
    {
        static_assert(N == 1 || N == 2, "");
        const float s = add(swap32(v[0], v[N - 1]));
        return sum16(add(swap16(s, s)));
    }
    template <int N> static __device__ __forceinline__ void unfold(float s, float (&v)[N])
    {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, s), 32 * i));
    }
    // Of R registers that are the same in a wave's rows of lanes, lane l gets those of
    // wave l % 16 (zeros behind the last).
    template <int R> __device__ __forceinline__ void spread(float (&s)[R])
    {
        const int lane = lane_id(), row = lane >> 4, of = lane & 15;
        if (of == 0)
#pragma unroll
            for (int i = 0; i < R; ++i) red[round][i][row][wave_id()] = s[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < R; ++i) s[i] = of < waves ? red[round][i][row][of] : 0.f;
        round ^= 1;  // (one barrier each: the other round's values have been read by all when it is passed)
    }
    template <int N> __device__ __forceinline__ void sum(float (&v)[N])
    {
        float s[1] = {fold(v)};
        if (waves > 1) spread(s), s[0] = sum16(s[0]);
        unfold(s[0], v);
    }
};

// Statistics of one or two rows held eight columns a chunk, C chunks a lane.  A layer
// norm's take one barrier: each wave has the mean and squares of its own columns, and
// those of all follow from these (the squares around the mean of all are each wave's
// around its own and its columns times the squared distance of the two: Chan, Golub
// and LeVeque, 1983).  The mean of all first, behind a barrier of its own: 98 us for 95.
template <int C> struct Cols {
    int col[C], left[C];  // of a lane's chunks; left <= 0: behind the row
    int at[C];            // where it reads: a row's last, partial chunk at the row's last eight columns
    bool full;            // all chunks of the wave have eight columns
    float mine, of;       // columns of the lane's wave, and of wave l % 16 of the team
};
// MEANS: some may be a layer norm; without, xh is x rstd (and f in rstd).  TINY: some eps is
// below LEAST_VAR, so that rows may have to be taken 2^100 fold: kernels of their own, since the
// others would pay in registers (join backward of 8192x4096 in bf16 with two rms norms 110 us for
// 99, two layer norms 122 for 115; norm backward with rms 50 for 50, of 4096x5003 42 for 38;
// forward the same).  TINY is with MEANS.
template <bool MEANS> __device__ __forceinline__ float xh_of(const Stat &s, float x) { return MEANS ? s.xh(x) : x * s.rstd; }
template <bool MEANS, bool TINY> __device__ __forceinline__ float dx_of(const BackStat &b, float g, float xh)
{
    return TINY ? b.dx_any(g, xh) : MEANS ? b.dx(g, xh) : __builtin_fmaf(-xh, b.m1, g) * b.s.rstd;
}
template <bool MEANS, bool TINY, int N, int C>
__device__ __forceinline__ void team_stats(Team &team, const Cols<C> &k, float by, const NormOf *const (&nm)[N], const float *const (&x)[N],
                                           Stat (&out)[N])
{
    bool layer = false;
    float m[N], v[N];  // means, squares around them
#pragma unroll
    for (int q = 0; q < N; ++q) layer |= MEANS && nm[q]->kind == DBS_NORM_LAYER, out[q] = Stat{1.f, 0.f, 0.f}, m[q] = 0.f;
    const float by_mine = MEANS ? 1.f / fmaxf(k.mine, 1.f) : 0.f;
    auto squares = [&](bool masked, bool plain) {
#pragma unroll
        for (int q = 0; q < N; ++q) {
            v[q] = 0.f;
#pragma unroll
            for (int i = 0; i < 8 * C; ++i) {
                float d = plain ? x[q][i] : __builtin_fmaf(x[q][i], out[q].f, -m[q]);
                if (masked && (i & 7) >= k.left[i >> 3]) d = 0.f;
                v[q] = __builtin_fmaf(d, d, v[q]);
            }
        }
    };
    // (without means, zeros stand behind the row)
    const bool masked = layer && !k.full;
    for (bool first = true;; first = false) {
        float s[2];  // the wave's own, which take no barrier
        if (layer) {
#pragma unroll
            for (int q = 0; q < N; ++q) {
                m[q] = 0.f;
                if (nm[q]->kind == DBS_NORM_LAYER)
#pragma unroll
                    for (int i = 0; i < 8 * C; ++i) m[q] = __builtin_fmaf(x[q][i], by_mine * out[q].f, m[q]);
            }
            s[1] = team.fold(m), team.unfold(s[1], m);
        }
        if (masked) squares(true, false);
        else if (!MEANS && first) squares(false, true);
        else squares(false, false);
        s[0] = team.fold(v);
        if (team.waves > 1) {
            if (layer) {
                // the waves' together: the mean of all, and for each wave its distance from that
                team.spread(s);
                const float mean = sum16(s[1] * (k.of * by)), d = s[1] - mean;
                s[0] = sum16(__builtin_fmaf(k.of * d, d, s[0])), s[1] = mean;
                team.unfold(s[1], m);
            } else {
                float t[1] = {s[0]};
                team.spread(t), s[0] = sum16(t[0]);
            }
        }
        team.unfold(s[0], v);
        bool again = false;
#pragma unroll
        for (int q = 0; q < N; ++q) {
            const float var = v[q] * by;
            out[q].mean = m[q];
            if constexpr (TINY) {
                if (out[q].f == 1.f) out[q].f = again_by(var, nm[q]->eps, m[q]), again |= out[q].f != 1.f;
            } else if (var > 3.402823466e38f && out[q].f == 1.f) out[q].f = DOWN, again = true;
            out[q].rstd = rsqrtf(var + nm[q]->eps * out[q].f * out[q].f);
        }
        if (__builtin_amdgcn_readfirstlane(again)) continue;  // (the same for the whole team)
        if (!MEANS)
#pragma unroll
            for (int q = 0; q < N; ++q) out[q].rstd *= out[q].f;
        return;
    }
}

// Column `col` of a row: an offset of 32 bits from an address that all lanes share.
template <class T> __device__ __forceinline__ T *at_col(T *row, int col)
{
    const uint32_t off = (uint32_t)col * (uint32_t)sizeof(T);
    return (T *)((char *)row + off);
}
__device__ __forceinline__ void put_floats(float *to, int left, const float *v, int at)
{
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < left) to[i] = v[at + i];
}
// Chunk c of a lane into a row.
template <class X, int C> __device__ __forceinline__ void put_chunk(void *base, int64_t ld, int64_t row, const Cols<C> &k, int c, const float (&v)[8])
{
    typename X::T *p = (typename X::T *)base + row * ld;
    if (k.full) put_eight<X>(at_col(p, k.col[c]), 8, v);
    else put_eight<X>(p + k.col[c], k.left[c], v);
}

// Which of a row's chunks a lane has, and which rows a team.
template <int C> struct Share : Cols<C> {
    int row, step;
    __device__ __forceinline__ Share(int n, int waves)
    {
        const int at = waves == 1 ? lane_id() : (int)threadIdx.x, teams = waves == 1 ? (int)blockDim.x / 64 : 1;
        row = __builtin_amdgcn_readfirstlane((int)blockIdx.x * teams + (waves == 1 ? wave_id() : 0));
        step = (int)gridDim.x * teams;
#pragma unroll
        for (int i = 0; i < C; ++i) this->col[i] = 8 * (i * 64 * waves + at), this->left[i] = n - this->col[i];
        bool ragged = false;
#pragma unroll
        for (int i = 0; i < C; ++i) this->at[i] = min(this->col[i], n - 8), ragged |= this->left[i] < 8;
        this->full = ballot(ragged) == 0;
        auto columns = [&](int wave) {
            int all = 0;
#pragma unroll
            for (int i = 0; i < C; ++i) all += wave < waves ? min(512, max(0, n - 512 * (i * waves + wave))) : 0;
            return (float)all;
        };
        this->mine = columns(waves == 1 ? 0 : wave_id()), this->of = columns(lane_id() & 15);
    }
};
typedef uint32_t v4u_t __attribute__((ext_vector_type(4)));
template <class X, int C> struct Chunks {
    typename X::V8 v[C];
    // A partial chunk comes as the row's last eight columns, in one load as the others:
    // parts of 4, 2 and 1 are put together behind a wait of their own, which the whole
    // team then meets at its next barrier (join backward of 4096x5119 in fp16 145 ->
    // 116 us, x5004 139 -> 107, x5003 119 -> 112).  It is settled where the row is used.
    __device__ __forceinline__ void load(const void *base, int64_t ld, int64_t row, const Cols<C> &k)
    {
        const typename X::T *p = (const typename X::T *)base + row * ld;
#pragma unroll
        for (int i = 0; i < C; ++i) v[i] = load_eight<X>(at_col(p, k.at[i]));
    }
    // A partial chunk moved down to its place, zeros behind it.
    __device__ __forceinline__ void settle(const Cols<C> &k)
    {
        if (k.full) return;
        auto pick = [](uint32_t mask, uint32_t there, uint32_t here) { return (there & mask) | (here & ~mask); };
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const v4u_t w = __builtin_bit_cast(v4u_t, v[i]);
            uint32_t w0 = w[0], w1 = w[1], w2 = w[2], w3 = w[3];
            const uint32_t by = 8 - max(0, min(8, k.left[i])), by4 = 0u - (by >> 2 & 1), by2 = 0u - (by >> 1 & 1), some = 0u - (by < 8);
            w0 = pick(by4, w2, w0), w1 = pick(by4, w3, w1), w2 &= ~by4, w3 &= ~by4;
            w0 = pick(by2, w1, w0), w1 = pick(by2, w2, w1), w2 = pick(by2, w3, w2), w3 &= ~by2;
            const uint32_t bits = 16 * (by & 1);
            const v4u_t z = {__builtin_amdgcn_alignbit(w1, w0, bits) & some, __builtin_amdgcn_alignbit(w2, w1, bits) & some,
                             __builtin_amdgcn_alignbit(w3, w2, bits) & some, w3 >> bits & some};
            v[i] = __builtin_bit_cast(typename X::V8, z);
        }
    }
    __device__ __forceinline__ void vector(const void *p, const Cols<C> &k, float none)
    {
#pragma unroll
        for (int i = 0; i < C; ++i) v[i] = get_vector<X>(k.left[i] > 0 ? p : nullptr, k.col[i], k.left[i], none);
    }
    __device__ __forceinline__ float operator[](int i) const { return (float)v[i >> 3][i & 7]; }
    // (to be taken apart where it is used: values that stay over the rows would
    // otherwise be held in 32 bits each)
    __device__ __forceinline__ void hold()
    {
#pragma unroll
        for (int i = 0; i < C; ++i) {
            v4u_t w = __builtin_bit_cast(v4u_t, v[i]);
            asm volatile("" : "+v"(w));
            v[i] = __builtin_bit_cast(typename X::V8, w);
        }
    }
};

// Each team takes rows of up to 512 C columns a wave, the next one on its way while
// one is worked on; the vectors stay in registers, or (C = 2, which needs those
// for the rows) come from the caches each time.  Bound by the bytes (join of 8192x4096
// in bf16 between two norms, with dropout: 57 us, 4.7 TB/s); a row or a few by the
// launch and one memory latency after the other (norm of 1x4096: 3.0 us).
template <class X, bool BRANCH, bool AFTER, bool BEFORE, bool TINY, int C>
__global__ __launch_bounds__(64 * MAX_TEAM) void k_edge(EdgeArgs a, int waves)
{
    __shared__ float red[2][2][4][MAX_TEAM];
    Team team{red, waves, 0};
    const Share<C> k(a.n, waves);
    uint64_t seed, offset;
    rng_of(a.drop, seed, offset);
    const int64_t chunks = (a.n + 7) / 8;
    const int last = (int)e8_blocks(a.n) * 16;
    const float by = 1.f / (float)a.n;
    Chunks<X, C> wa, ba, wb, bb, gate;
    auto vectors_before = [&]() {
        if constexpr (BEFORE) wb.vector(a.before.w, k, 1.f), bb.vector(a.before.b, k, 0.f);
    };
    auto vectors = [&]() {
        if constexpr (AFTER) wa.vector(a.after.w, k, 1.f), ba.vector(a.after.b, k, 0.f);
        if constexpr (BRANCH) gate.vector(a.ldg == 0 ? a.gate : nullptr, k, 1.f);
    };
    if (C == 1) vectors(), vectors_before();
    const bool gates = BRANCH && a.gate && a.ldg != 0;
    Chunks<X, C> res, branch, gnext;
    auto load = [&](int row) {
        res.load(a.res, a.ldr, row, k);
        if constexpr (BRANCH) {
            branch.load(a.branch, a.ldb, row, k);
            if (gates) gnext.load(a.gate, a.ldg, row, k);
        }
    };
    // (where registers are left for it: two chunks a lane of a join have none, and take their
    // vectors only where they are used; 2048x14336 in bf16 with two layer norms 109 -> 80 us,
    // with one norm 57 to 59 -> 41 to 45)
    constexpr bool AHEAD = C == 1 || !BRANCH;
    if (AHEAD && k.row < a.rows) load(k.row);
    for (int row = k.row; row < a.rows; row += k.step) {
        if (!AHEAD) load(row);
        res.settle(k);
        if constexpr (BRANCH) {
            branch.settle(k);
            if (gates) gnext.settle(k);
        }
        float s[8 * C], u[8 * C];
#pragma unroll
        for (int i = 0; i < 8 * C; ++i) {
            s[i] = res[i];
            if constexpr (BRANCH) u[i] = branch[i];
        }
        const Chunks<X, C> now = gnext;
        if (AHEAD && row + k.step < a.rows) load(row + k.step);
        if constexpr (BRANCH) {
            if constexpr (AFTER) {
                const NormOf *nm[1] = {&a.after};
                const float *x[1] = {u};
                Stat st[1];
                team_stats<true, TINY>(team, k, by, nm, x, st);
                if (C > 1) vectors();
#pragma unroll
                for (int i = 0; i < 8 * C; ++i) u[i] = __builtin_fmaf(st[0].xh(u[i]), wa[i], ba[i]);
            } else if (C > 1) vectors();
            if (gates) gate = now;
            // (the next row is taken as arrived here, before this one's stores, which the
            // same counter counts: later the wait would be for them)
            if (AHEAD) {
                res.hold(), branch.hold();
                if (gates) gnext.hold();
            }
#pragma unroll
            for (int c = 0; c < C; ++c) {
                if (a.drop.threshold) {
                    float v[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = u[8 * c + i];
                    drop_eight(a.drop, seed, offset, row * chunks + k.col[c] / 8, v);
#pragma unroll
                    for (int i = 0; i < 8; ++i) u[8 * c + i] = v[i];
                }
                float out[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) out[i] = s[8 * c + i] = __builtin_fmaf(gate[8 * c + i], u[8 * c + i], a.scale * s[8 * c + i]);
                if (!k.full)  // (zeros behind the row, as everywhere)
#pragma unroll
                    for (int i = 0; i < 8; ++i) s[8 * c + i] = i < k.left[c] ? s[8 * c + i] : 0.f;
                put_chunk<X, C>(a.stream, a.lds, row, k, c, out);
            }
        }
        if constexpr (BEFORE) {
            const NormOf *nm[1] = {&a.before};
            const float *x[1] = {s};
            Stat st[1];
            team_stats<true, TINY>(team, k, by, nm, x, st);
            if (C > 1) vectors_before();
            if (AHEAD && !BRANCH) res.hold();
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float h[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) h[i] = __builtin_fmaf(st[0].xh(s[8 * c + i]), wb[8 * c + i], bb[8 * c + i]);
                if (a.codes) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) h[i] = i < k.left[c] ? h[i] : 0.f;
                    put_codes<X>(a, row, k.col[c] / 8, last, h);
                } else put_chunk<X, C>(a.h, a.ldh, row, k, c, h);
            }
        }
    }
}

// One row's chunk of the backward pass: what it reads, and what follows from it.
template <class X, bool BRANCH> struct BackChunk {
    float dh[8], xb[8], d[8], g[8];       // gradient of h, normalised stream, ds*, dh w
    float ub[8], keep[8], gate[8], du[8]; // normalised branch or branch, what dropout multiplies by, gradient behind the norm
};
// The part up to ds* (everything that `before` needs: its statistics, and with
// `means` its two means).
template <class X, bool BRANCH>
__device__ __forceinline__ void back_before(const EdgeBackArgs &a, int64_t row, int col, int left, const BackStat &b, bool means,
                                            BackChunk<X, BRANCH> &k)
{
    typedef typename X::T T;
    if (a.ds) get_floats<X>((const T *)a.ds + row * a.ldds + col, left, k.d);
    else
#pragma unroll
        for (int i = 0; i < 8; ++i) k.d[i] = 0.f;
    if (a.before.kind == DBS_NORM_NONE) return;
    get_floats<X>((const T *)a.dh + row * a.lddh + col, left, k.dh);
    get_floats<X>((const T *)a.stream + row * a.lds + col, left, k.xb);
    const typename X::V8 w = get_vector<X>(a.before.w, col, left, 1.f);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        k.xb[i] = b.s.xh(k.xb[i]);
        k.g[i] = k.dh[i] * (float)w[i];
        if (means) k.d[i] += b.dx_any(k.g[i], k.xb[i]);
    }
}
// The part from ds* to the gradient behind `after` (with `means` through it).
template <class X, bool BRANCH>
__device__ __forceinline__ void back_after(const EdgeBackArgs &a, int64_t row, int col, int left, uint64_t seed, uint64_t offset,
                                           const BackStat &f, BackChunk<X, BRANCH> &k)
{
    typedef typename X::T T;
    const int64_t chunks = (a.n + 7) / 8;
    if (a.branch) get_floats<X>((const T *)a.branch + row * a.ldb + col, left, k.ub);
    const typename X::V8 g = get_vector<X>(a.gate ? (const T *)a.gate + row * a.ldg : nullptr, col, left, 1.f);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        k.keep[i] = 1.f;
        k.gate[i] = (float)g[i];
        if (a.after.kind != DBS_NORM_NONE) k.ub[i] = f.s.xh(k.ub[i]);
    }
    if (a.drop.threshold) drop_eight(a.drop, seed, offset, row * chunks + col / 8, k.keep);
#pragma unroll
    for (int i = 0; i < 8; ++i) k.du[i] = k.keep[i] != 0.f ? k.d[i] * k.gate[i] * k.keep[i] : 0.f;
}

// The statistics and means of each row.
template <class X, bool BRANCH> __global__ __launch_bounds__(64 * LONG_WAVES) void k_edge_back_rows(EdgeBackArgs a)
{
    typedef typename X::T T;
    __shared__ float red[2][LONG_WAVES];
    GroupSum<LONG_WAVES> total{red};
    uint64_t seed, offset;
    rng_of(a.drop, seed, offset);
    const float by = 1.f / (float)a.n;
    for (int row = (int)blockIdx.x; row < a.rows; row += (int)gridDim.x) {
        BackStat b{}, f{};
        if (a.before.kind != DBS_NORM_NONE) {
            const T *x = (const T *)a.stream + row * a.lds;
            b.s = row_stat(a.before, a.n, total, [&](int c, float(&v)[8]) { get_floats<X>(x + 8 * c, a.n - 8 * c, v); });
            double m1 = 0.0, m2 = 0.0;  // (as in row_stat)
            for (int c = (int)threadIdx.x; 8 * c < a.n; c += 64 * LONG_WAVES) {
                BackChunk<X, BRANCH> k;
                back_before(a, row, 8 * c, a.n - 8 * c, b, false, k);
                float s1 = 0.f, s2 = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (8 * c + i < a.n) s1 = __builtin_fmaf(k.g[i], k.xb[i], s1), s2 += k.g[i];
                m1 += s1, m2 += s2;
            }
            b.m1 = total((float)m1) * by;
            if (a.before.kind == DBS_NORM_LAYER) b.m2 = total((float)m2) * by;
        }
        if (BRANCH && a.after.kind != DBS_NORM_NONE) {
            const T *x = (const T *)a.branch + row * a.ldb;
            f.s = row_stat(a.after, a.n, total, [&](int c, float(&v)[8]) { get_floats<X>(x + 8 * c, a.n - 8 * c, v); });
            double m1 = 0.0, m2 = 0.0;
            for (int c = (int)threadIdx.x; 8 * c < a.n; c += 64 * LONG_WAVES) {
                BackChunk<X, BRANCH> k;
                const int left = a.n - 8 * c;
                back_before(a, row, 8 * c, left, b, true, k);
                back_after(a, row, 8 * c, left, seed, offset, f, k);
                const typename X::V8 w = get_vector<X>(a.after.w, 8 * c, left, 1.f);
                float s1 = 0.f, s2 = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float g = k.du[i] * (float)w[i];
                    if (i < left) s1 = __builtin_fmaf(g, k.ub[i], s1), s2 += g;
                }
                m1 += s1, m2 += s2;
            }
            f.m1 = total((float)m1) * by;
            if (a.after.kind == DBS_NORM_LAYER) f.m2 = total((float)m2) * by;
        }
        if (threadIdx.x == 0) a.stat[2 * (int64_t)row] = b, a.stat[2 * (int64_t)row + 1] = f;
    }
}

// Everything else: a workgroup has a strip of 512 columns and a range of rows,
// a lane eight columns, whose sums it holds.  Both kernels read a row again, from the caches at
// best: join backward of 2048x14336 in bf16 with an rms norm before 128 us, with two layer
// norms 257, a copy of the bytes of one reading 61 and 73.
constexpr int STRIP = 512, STRIP_WAVES = 4;
__host__ __device__ __forceinline__ int first_row(int64_t rows, int blocks, int block) { return (int)(rows * block / blocks); }

template <class X, bool BRANCH> __global__ __launch_bounds__(64 * STRIP_WAVES) void k_edge_back_strip(EdgeBackArgs a)
{
    typedef typename X::T T;
    __shared__ float part[STRIP_WAVES][STRIP];
    const int lane = lane_id(), wave = wave_id();
    const int64_t col64 = (int64_t)blockIdx.x * STRIP + 8 * lane;
    const int col = (int)min(col64, (int64_t)a.n), left = a.n - col, block = (int)blockIdx.y;
    uint64_t seed, offset;
    rng_of(a.drop, seed, offset);
    const int r1 = first_row(a.rows, a.blocks, block + 1);
    float sum[SUMS][8] = {};
    const typename X::V8 wa = get_vector<X>(left > 0 ? a.after.w : nullptr, col, left, 1.f);
    const typename X::V8 ba = get_vector<X>(left > 0 ? a.after.b : nullptr, col, left, 0.f);
    for (int row = first_row(a.rows, a.blocks, block) + wave; row < r1 && left > 0; row += STRIP_WAVES) {
        BackStat b{}, f{};
        if (a.stat) b = a.stat[2 * (int64_t)row], f = a.stat[2 * (int64_t)row + 1];
        BackChunk<X, BRANCH> k;
        back_before(a, row, col, left, b, true, k);
        if (a.before.kind != DBS_NORM_NONE)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                sum[SUM_BEFORE_W][i] = __builtin_fmaf(k.dh[i], k.xb[i], sum[SUM_BEFORE_W][i]);
                sum[SUM_BEFORE_B][i] += k.dh[i];
            }
        if (a.dres) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = k.d[i] * a.scale;
            put_eight<X>((T *)a.dres + row * a.lddr + col, left, v);
        }
        if constexpr (BRANCH) {
            back_after(a, row, col, left, seed, offset, f, k);
            if (a.gate) {
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float u = a.after.kind != DBS_NORM_NONE ? __builtin_fmaf(k.ub[i], (float)wa[i], (float)ba[i]) : k.ub[i];
                    v[i] = k.keep[i] != 0.f ? k.d[i] * u * k.keep[i] : 0.f;
                    sum[SUM_GATE][i] += v[i];
                }
                if (a.dgate) put_eight<X>((T *)a.dgate + row * a.lddg + col, left, v);
            }
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[i] = k.du[i];
                if (a.after.kind != DBS_NORM_NONE) {
                    sum[SUM_AFTER_W][i] = __builtin_fmaf(v[i], k.ub[i], sum[SUM_AFTER_W][i]);
                    sum[SUM_AFTER_B][i] += v[i];
                    v[i] = f.dx_any(v[i] * (float)wa[i], k.ub[i]);
                }
            }
            if (a.dbranch) put_eight<X>((T *)a.dbranch + row * a.lddb + col, left, v);
        }
    }
#pragma unroll
    for (int q = 0; q < SUMS; ++q) {
        if (a.at[q] < 0) continue;
#pragma unroll
        for (int i = 0; i < 8; ++i) part[wave][8 * lane + i] = sum[q][i];
        __syncthreads();
        for (int c = (int)threadIdx.x; c < STRIP; c += 64 * STRIP_WAVES) {
            const int64_t at = (int64_t)blockIdx.x * STRIP + c;
            if (at >= a.n) continue;
            float s = part[0][c];
#pragma unroll
            for (int w = 1; w < STRIP_WAVES; ++w) s += part[w][c];
            a.part[((int64_t)block * a.sums + a.at[q]) * a.n + at] = s;
        }
        __syncthreads();
    }
}

// The kernel's arguments (its first), read anew from here on: kept over the rows, the
// many of them take more scalar registers than there are, and each use a lane's read
// (join backward of 4096x5003 in fp16 109 -> 102 us).
template <class A> using Args4 = const __attribute__((address_space(4))) A;
template <class A> __device__ __forceinline__ Args4<A> *args_again()
{
    auto *p = (Args4<A> *)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return p;
}
template <class N> __device__ __forceinline__ NormOf norm_of(N &n) { return NormOf{n.kind, n.eps, n.w, n.b}; }

// Waves of a SIMD whose registers the compiler is to fit.  With one norm at most two
// teams of eight waves run on a compute unit (join backward with a layer norm after,
// gate and dropout, 4096x4096 in bf16: 54 us; with one team's registers 62); those of
// both norms do not fit into as few (196 for 89).
constexpr int back_simd(int team, int chunks, bool both) { return team == 8 && chunks == 1 && !both ? 4 : team / 4; }

// The same for the gradients: a lane holds the sums over its team's rows of its
// columns, the workgroups' are added afterwards.  A norm alone is bound by the bytes
// (8192x4096 in bf16: 52 us, 5.2 TB/s), a join with an rms norm before nearly (4096x4096
// in bf16: 37 us with the sums' end, a copy of as many bytes 35); one with both norms by the
// vector ALUs, some 600 instructions for a wave's 64 chunks, and by the three barriers of
// a row (4096x4096 in bf16 with layer norms 70 us, fp16 rows of 5003 92; a copy 42 and 51).
template <class X, bool BRANCH, bool AFTER, bool BEFORE, bool MEANS, bool TINY, int C, int TEAM>
__global__ __launch_bounds__(64 * TEAM, back_simd(TEAM, C, AFTER && BEFORE)) void k_edge_back(EdgeBackArgs a, int waves)
{
    __shared__ float red[2][2][4][MAX_TEAM], lanes[4][C * 512];
    Team team{red, waves, 0};
    const Share<C> k(a.n, waves);
    uint64_t seed, offset;
    rng_of(a.drop, seed, offset);
    const int64_t chunks = (a.n + 7) / 8;
    const float by = 1.f / (float)a.n;
    const bool gates = BRANCH && a.gate && a.ldg != 0, dgates = BRANCH && a.gate && (a.dgate || a.at[SUM_GATE] >= 0);
    Chunks<X, C> wa, ba, wb, gate;
    auto vectors = [&]() {
        if constexpr (BEFORE) wb.vector(a.before.w, k, 1.f);
        if constexpr (AFTER) wa.vector(a.after.w, k, 1.f), ba.vector(dgates ? a.after.b : nullptr, k, 0.f);
        if constexpr (BRANCH) gate.vector(a.ldg == 0 ? a.gate : nullptr, k, 1.f);
    };
    vectors();
    float sum[BRANCH ? SUMS : 2][8 * C] = {};
    Chunks<X, C> nds{}, ndh, nxs, nxu{};
    auto load = [&](int row) {
        const auto &a = *args_again<EdgeBackArgs>();
        if (a.ds) nds.load(a.ds, a.ldds, row, k);
        if constexpr (BEFORE) ndh.load(a.dh, a.lddh, row, k), nxs.load(a.stream, a.lds, row, k);
        if constexpr (BRANCH)
            if (a.branch) nxu.load(a.branch, a.ldb, row, k);
    };
    constexpr bool AHEAD = C == 1;  // (two chunks a lane leave no registers for it)
    if (AHEAD && k.row < a.rows) load(k.row);
    for (int row = k.row; row < a.rows; row += k.step) {
        if (!AHEAD) load(row);
        nds.settle(k), ndh.settle(k), nxs.settle(k), nxu.settle(k);
        const Chunks<X, C> dh = ndh;
        const auto &a = *args_again<EdgeBackArgs>();
        if constexpr (TEAM > 8 || C > 1 || (BRANCH && !(AFTER && BEFORE))) {
            if constexpr (BEFORE) wb.hold();
            if constexpr (AFTER) wa.hold(), ba.hold();
            if constexpr (BRANCH) gate.hold();
        }
        if constexpr (BRANCH)
            if (gates) gate.load(a.gate, a.ldg, row, k), gate.settle(k);
        float d[8 * C], xb[8 * C], u[8 * C];
        Stat sb{}, sa{};
#pragma unroll
        for (int i = 0; i < 8 * C; ++i) {
            d[i] = nds[i];
            if (BEFORE) xb[i] = nxs[i];
            if (BRANCH) u[i] = nxu[i];
        }
        if (AHEAD && row + k.step < a.rows) load(row + k.step);
        if constexpr (AFTER && BEFORE) {
            const NormOf before = norm_of(a.before), after = norm_of(a.after), *nm[2] = {&before, &after};
            const float *x[2] = {xb, u};
            Stat st[2];
            team_stats<MEANS, TINY>(team, k, by, nm, x, st);
            sb = st[0], sa = st[1];
        } else if constexpr (AFTER || BEFORE) {
            const NormOf one = norm_of(BEFORE ? a.before : a.after), *nm[1] = {&one};
            const float *x[1] = {BEFORE ? xb : u};
            Stat st[1];
            team_stats<MEANS, TINY>(team, k, by, nm, x, st);
            (BEFORE ? sb : sa) = st[0];
        }
        if constexpr (BEFORE) {
            float m[MEANS ? 2 : 1] = {};
#pragma unroll
            for (int i = 0; i < 8 * C; ++i) {
                xb[i] = xh_of<MEANS>(sb, xb[i]);
                const float g = dh[i] * wb[i];
                m[0] = __builtin_fmaf(g, xb[i], m[0]);
                if (MEANS) m[MEANS] += g;
                sum[SUM_BEFORE_W][i] = __builtin_fmaf(dh[i], xb[i], sum[SUM_BEFORE_W][i]);
            }
            if (a.at[SUM_BEFORE_B] >= 0)
#pragma unroll
                for (int i = 0; i < 8 * C; ++i) sum[SUM_BEFORE_B][i] += dh[i];
            team.sum(m);
            const BackStat b{sb, m[0] * by, MEANS && a.before.kind == DBS_NORM_LAYER ? m[MEANS] * by : 0.f};
#pragma unroll
            for (int i = 0; i < 8 * C; ++i) d[i] += dx_of<MEANS, TINY>(b, dh[i] * wb[i], xb[i]);
        }
        // (the next row is taken as arrived here, before this one's stores, which the
        // same counter counts: later the wait would be for them)
        if (AHEAD) {
            if (a.ds) nds.hold();
            if constexpr (BEFORE) ndh.hold(), nxs.hold();
            if constexpr (BRANCH) nxu.hold();
        }
        if (a.dres)
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = d[8 * c + i] * a.scale;
                put_chunk<X, C>(a.dres, a.lddr, row, k, c, v);
            }
        if constexpr (BRANCH) {
            const auto &a = *args_again<EdgeBackArgs>();
            float m[MEANS ? 2 : 1] = {};
#pragma unroll
            for (int c = 0; c < C; ++c) {
                uint32_t kept = 255u;
                if (a.drop.threshold) kept = kept_of(a.drop.threshold, seed, offset, row * chunks + k.col[c] / 8);
                const float by_kept = a.drop.threshold ? a.drop.scale : 1.f;
                if constexpr (AFTER)
#pragma unroll
                    for (int i = 0; i < 8; ++i) u[8 * c + i] = xh_of<MEANS>(sa, u[8 * c + i]);
                if (dgates) {
                    float v[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int q = 8 * c + i;
                        const float y = AFTER ? __builtin_fmaf(u[q], wa[q], ba[q]) : u[q];
                        v[i] = kept >> i & 1 ? d[q] * y * by_kept : 0.f;
                        sum[SUM_GATE][q] += v[i];
                    }
                    if (a.dgate) put_chunk<X, C>(a.dgate, a.lddg, row, k, c, v);
                }
                // (behind dropout and gate)
                if (a.gate)
#pragma unroll
                    for (int i = 0; i < 8; ++i) d[8 * c + i] *= gate[8 * c + i];
                if (a.drop.threshold)
#pragma unroll
                    for (int i = 0; i < 8; ++i) d[8 * c + i] = kept >> i & 1 ? d[8 * c + i] * by_kept : 0.f;
                if (!k.full)
#pragma unroll
                    for (int i = 0; i < 8; ++i) d[8 * c + i] = i < k.left[c] ? d[8 * c + i] : 0.f;
                if constexpr (AFTER) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int q = 8 * c + i;
                        const float g = d[q] * wa[q];
                        m[0] = __builtin_fmaf(g, u[q], m[0]);
                        if (MEANS) m[MEANS] += g;
                        sum[SUM_AFTER_W][q] = __builtin_fmaf(d[q], u[q], sum[SUM_AFTER_W][q]);
                    }
                    if (a.at[SUM_AFTER_B] >= 0)
#pragma unroll
                        for (int i = 0; i < 8; ++i) sum[SUM_AFTER_B][8 * c + i] += d[8 * c + i];
                }
            }
            if constexpr (AFTER) {
                team.sum(m);
                const BackStat b{sa, m[0] * by, MEANS && a.after.kind == DBS_NORM_LAYER ? m[MEANS] * by : 0.f};
#pragma unroll
                for (int i = 0; i < 8 * C; ++i) d[i] = dx_of<MEANS, TINY>(b, d[i] * wa[i], u[i]);
            }
            if (a.dbranch)
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    float v[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = d[8 * c + i];
                    put_chunk<X, C>(a.dbranch, a.lddb, row, k, c, v);
                }
        }
    }
#pragma unroll
    for (int q = 0; q < (BRANCH ? SUMS : 2); ++q) {
        if (a.at[q] < 0) continue;
        float *to = a.part + ((int64_t)blockIdx.x * a.sums + a.at[q]) * a.n;
        if (waves == 1) {  // a workgroup's four teams are waves: their sums are added here
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 8 * C; ++i) lanes[wave_id()][k.col[i >> 3] + (i & 7)] = sum[q][i];
            __syncthreads();
            for (int c = (int)threadIdx.x; c < a.n; c += (int)blockDim.x) to[c] = lanes[0][c] + lanes[1][c] + lanes[2][c] + lanes[3][c];
        } else
#pragma unroll
            for (int c = 0; c < C; ++c) put_floats(to + k.col[c], k.left[c], sum[q], 8 * c);
    }
}
// The workgroups' sums, in their order: a column a lane, the workgroups shared
// out to the waves.
constexpr int TOTAL_WAVES = 16;
struct TotalArgs {
    const float *part;
    void *out[SUMS];
    int32_t sums, blocks, n, first;
};
template <class X> __global__ __launch_bounds__(64 * TOTAL_WAVES) void k_edge_total(TotalArgs a)
{
    __shared__ float part[TOTAL_WAVES][64];
    const int lane = lane_id(), wave = wave_id(), q = (int)blockIdx.y;
    const int64_t c = ((int64_t)blockIdx.x + a.first) * 64 + lane;
    float s = 0.f;
    if (c < a.n)
#pragma unroll 4
        for (int i = wave; i < a.blocks; i += TOTAL_WAVES) s += a.part[((int64_t)i * a.sums + q) * a.n + c];
    part[wave][lane] = s;
    __syncthreads();
    if (wave != 0 || c >= a.n) return;
#pragma unroll
    for (int w = 1; w < TOTAL_WAVES; ++w) s += part[w][lane];
    ((typename X::T *)a.out[q])[c] = (typename X::T)s;
}

// ---------------------------------------------------------------------------
// dropout alone
// ---------------------------------------------------------------------------
constexpr int DROP_TPB = 256;

// A thread takes chunks of eight columns, its next one a whole grid on.  Bound by
// the bytes; 16 random bits an element keep the generator's products (two for each of
// ten rounds) to two and a half an element, which the vector ALUs do beside them
// (16384x4096 in bf16: 42 us, 6.4 TB/s, a copy of as much 55 in HBM alone: part of it
// stays in the last-level cache).
template <class X>
__global__ __launch_bounds__(DROP_TPB) void k_dropout(const typename X::T *x, int64_t ldx, int32_t rows, int32_t n, int32_t per,
                                                      Drop d, typename X::T *y, int64_t ldy)
{
    uint64_t seed, offset;
    rng_of(d, seed, offset);
    const int64_t chunks = (int64_t)rows * per;
    for (int64_t c = (int64_t)blockIdx.x * DROP_TPB + threadIdx.x; c < chunks; c += (int64_t)gridDim.x * DROP_TPB) {
        const int64_t row = chunks <= UINT32_MAX ? (uint32_t)c / (uint32_t)per : c / per;  // (32 bits divide much faster)
        const int col = 8 * (int)(c - row * per), left = n - col;
        float v[8];
        get_floats<X>(x + row * ldx + col, left, v);
        if (d.threshold) drop_eight(d, seed, offset, c, v);
        put_eight<X>(y + row * ldy + col, left, v);
    }
}

// ---------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------
// A team's waves for rows of n columns, C chunks a lane; workgroups of one team, or of
// four of a wave each.
static int team_waves(int32_t n, int c) { return (int)(((int64_t)n + 512 * c - 1) / (512 * c)); }
static int team_threads(int waves) { return 64 * (waves == 1 ? 4 : waves); }
static int team_rows(int waves) { return waves == 1 ? 4 : 1; }

// Whether some norm's eps is below LEAST_VAR.
static bool any_tiny(const NormOf &after, const NormOf &before)
{
    return (after.kind != DBS_NORM_NONE && after.eps < LEAST_VAR) || (before.kind != DBS_NORM_NONE && before.eps < LEAST_VAR);
}

template <class X, bool BRANCH, bool AFTER, bool BEFORE, bool TINY> static hipError_t edge_t(const EdgeArgs &a, int32_t cus, hipStream_t s)
{
    if (a.n < 8 || a.n > 1024 * MAX_TEAM) {
        hipLaunchKernelGGL((k_edge_long<X, BRANCH>), dim3((unsigned)std::min(a.rows, 2 * cus)), dim3(64 * LONG_WAVES), 0, s, a);
        return hipGetLastError();
    }
    const int c = a.n <= 512 * MAX_TEAM ? 1 : 2, waves = team_waves(a.n, c), rows = team_rows(waves);
    // As many workgroups as run beside each other: four waves on a SIMD, of a norm alone
    // six.  (With eight for all, rounded up to whole teams: join of 8192x4096 in bf16 with
    // two layer norms 61 us for 59, 4096x5003 61 for 56; a norm of it 16.9 for 16.3, with
    // four 19.5.)
    const int64_t most = (int64_t)cus * std::max(1, (BRANCH ? 1024 : 1536) / team_threads(waves));
    const dim3 grid((unsigned)std::min<int64_t>(((int64_t)a.rows + rows - 1) / rows, most)), block((unsigned)team_threads(waves));
    if (c == 1) hipLaunchKernelGGL((k_edge<X, BRANCH, AFTER, BEFORE, TINY, 1>), grid, block, 0, s, a, waves);
    else hipLaunchKernelGGL((k_edge<X, BRANCH, AFTER, BEFORE, TINY, 2>), grid, block, 0, s, a, waves);
    return hipGetLastError();
}
template <class X, bool TINY> static hipError_t edge_n(const EdgeArgs &a, int32_t cus, hipStream_t s)
{
    const bool after = a.after.kind != DBS_NORM_NONE, before = a.before.kind != DBS_NORM_NONE;
    if (!a.branch) return edge_t<X, false, false, true, TINY>(a, cus, s);
    if (after) return before ? edge_t<X, true, true, true, TINY>(a, cus, s) : edge_t<X, true, true, false, TINY>(a, cus, s);
    return before ? edge_t<X, true, false, true, TINY>(a, cus, s) : edge_t<X, true, false, false, false>(a, cus, s);
}
template <class X> static hipError_t edge_x(const EdgeArgs &a, int32_t cus, hipStream_t s)
{
    return any_tiny(a.after, a.before) ? edge_n<X, true>(a, cus, s) : edge_n<X, false>(a, cus, s);
}
hipError_t launch_edge(bool bf16, const EdgeArgs &a, int32_t cus, hipStream_t s)
{
    if (a.rows == 0 || a.n == 0) return hipSuccess;
    return bf16 ? edge_x<Bf16>(a, cus, s) : edge_x<Fp16>(a, cus, s);
}

// The most rows that a lane adds up in a row: of 2^13 equal terms a sum in 32 bits may be off by
// half a step of fp16 (2^16 of them: 0.1%).
constexpr int64_t MOST_ROWS = 2048;
// Workgroups along the rows: enough to fill the device, none with less than a row
// for each wave.
static int32_t strip_blocks(int32_t rows, int32_t n, int32_t cus)
{
    const int64_t strips = ((int64_t)n + STRIP - 1) / STRIP, want = strips ? (4 * (int64_t)cus + strips - 1) / strips : 1;
    const int64_t least = ((int64_t)rows + STRIP_WAVES * MOST_ROWS - 1) / (STRIP_WAVES * MOST_ROWS);
    return (int32_t)std::max<int64_t>(1, std::min<int64_t>({std::max(want, least), ((int64_t)rows + STRIP_WAVES - 1) / STRIP_WAVES, 65535}));
}
// Rows of 8 (a load) up to 8192 columns (a norm alone: 16384) are held in registers: one chunk a
// lane, or, where 16 waves have no registers for the sums, two or four of eight waves.
static bool back_fits(bool branch, int32_t n) { return n >= 8 && n <= (branch ? 8192 : 16384); }
static int back_chunks(bool branch, int32_t n) { return branch ? (n > 6144 ? 2 : 1) : n > 8192 ? 4 : 1; }
// The most waves of a team that a kernel is made for: the fewer, the more registers
// each.  With both norms a team of up to four waves gets the registers of three on a
// SIMD, so that three run on a compute unit (8192x2048 in bf16 with two layer norms 84 ->
// 71 us; teams of five and six, which have two waves on one SIMD, would run alone as they do).
static int back_team(bool both, int waves, int chunks) { return chunks > 1 ? 8 : waves <= 8 && (!both || waves > 4) ? 8 : waves <= 12 ? 12 : 16; }
// Workgroups: as many as run beside each other, each with a few rows, since its sums'
// bytes are written and read again; but no compute unit is left without.  (A workgroup's
// waves go to the SIMDs in turn; one with five counts as one with eight.  More workgroups than
// that: 8192x2560 128 us for 107; fewer: 16384x1024 88 for 75.)
static int32_t back_groups(bool branch, bool both, int32_t rows, int32_t n, int32_t cus)
{
    const int chunks = back_chunks(branch, n), waves = team_waves(n, chunks), each = team_rows(waves), team = back_team(both, waves, chunks);
    const int simd = back_simd(team, chunks, both), beside = waves == 2 ? 2 * simd : simd / ((team_threads(waves) + 255) / 256);
    const int64_t teams = ((int64_t)rows + each - 1) / each;
    const int64_t groups = std::min(std::min(teams, (int64_t)cus * std::max(1, beside)), std::max<int64_t>(cus, (teams + 7) / 8));
    return (int32_t)std::max(groups, (teams + MOST_ROWS - 1) / MOST_ROWS);
}
static int32_t sum_blocks(bool branch, bool both, int32_t rows, int32_t n, int32_t cus)
{
    return back_fits(branch, n) ? back_groups(branch, both, rows, n, cus) : strip_blocks(rows, n, cus);
}
static size_t part_bytes(bool branch, bool both, int32_t rows, int32_t n, int sums, int32_t cus)
{
    return ((size_t)sum_blocks(branch, both, rows, n, cus) * sums * n * 4 + 255) / 256 * 256;
}
size_t edge_back_work(int32_t rows, int32_t n, int sums, int32_t cus)
{
    if (n == 0) return 0;
    const size_t part = std::max({part_bytes(false, false, rows, n, sums, cus), part_bytes(true, false, rows, n, sums, cus), part_bytes(true, true, rows, n, sums, cus)});
    return part + (back_fits(true, n) ? 0 : (size_t)rows * 2 * sizeof(BackStat));
}

template <class X> static hipError_t total_t(TotalArgs t, hipStream_t s)
{
    return launch_parts(((int64_t)t.n + 63) / 64, 64 * TOTAL_WAVES, [&](int32_t first, dim3 grid) {
        t.first = first;
        grid.y = (unsigned)t.sums;
        hipLaunchKernelGGL(k_edge_total<X>, grid, dim3(64 * TOTAL_WAVES), 0, s, t);
    });
}
template <class X, bool BRANCH, bool AFTER, bool BEFORE, bool MEANS, bool TINY> static void edge_back_m(const EdgeBackArgs &a, hipStream_t s)
{
    const int chunks = back_chunks(BRANCH, a.n), waves = team_waves(a.n, chunks), team = back_team(AFTER && BEFORE, waves, chunks);
    const dim3 grid((unsigned)a.blocks), block((unsigned)team_threads(waves));
    if (chunks > 1) hipLaunchKernelGGL((k_edge_back<X, BRANCH, AFTER, BEFORE, MEANS, TINY, BRANCH ? 2 : 4, 8>), grid, block, 0, s, a, waves);
    else if (team == 8) hipLaunchKernelGGL((k_edge_back<X, BRANCH, AFTER, BEFORE, MEANS, TINY, 1, 8>), grid, block, 0, s, a, waves);
    else if (team == 12) hipLaunchKernelGGL((k_edge_back<X, BRANCH, AFTER, BEFORE, MEANS, TINY, 1, 12>), grid, block, 0, s, a, waves);
    else if constexpr (!BRANCH) hipLaunchKernelGGL((k_edge_back<X, BRANCH, AFTER, BEFORE, MEANS, TINY, 1, 16>), grid, block, 0, s, a, waves);
}
template <class X, bool BRANCH, bool AFTER, bool BEFORE> static hipError_t edge_back_t(const EdgeBackArgs &a, int32_t cus, hipStream_t s)
{
    if (a.rows > 0 && back_fits(BRANCH, a.n)) {
        if constexpr (AFTER || BEFORE) {
            if (any_tiny(a.after, a.before)) edge_back_m<X, BRANCH, AFTER, BEFORE, true, true>(a, s);
            else if ((AFTER && a.after.kind == DBS_NORM_LAYER) || (BEFORE && a.before.kind == DBS_NORM_LAYER))
                edge_back_m<X, BRANCH, AFTER, BEFORE, true, false>(a, s);
            else edge_back_m<X, BRANCH, AFTER, BEFORE, false, false>(a, s);
        } else edge_back_m<X, BRANCH, AFTER, BEFORE, false, false>(a, s);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    } else if (a.rows > 0) {
        if (a.stat) hipLaunchKernelGGL((k_edge_back_rows<X, BRANCH>), dim3((unsigned)std::min(a.rows, 2 * cus)), dim3(64 * LONG_WAVES), 0, s, a);
        const dim3 grid((unsigned)(((int64_t)a.n + STRIP - 1) / STRIP), (unsigned)a.blocks);
        hipLaunchKernelGGL((k_edge_back_strip<X, BRANCH>), grid, dim3(64 * STRIP_WAVES), 0, s, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (!a.sums) return hipSuccess;
    TotalArgs t{a.part, {}, a.sums, a.rows > 0 ? a.blocks : 0, a.n, 0};
    for (int q = 0; q < SUMS; ++q)
        if (a.at[q] >= 0) t.out[a.at[q]] = a.sum[q];
    return total_t<X>(t, s);
}
template <class X> static hipError_t edge_back_x(const EdgeBackArgs &a, bool has_branch, int32_t cus, hipStream_t s)
{
    const bool after = a.after.kind != DBS_NORM_NONE, before = a.before.kind != DBS_NORM_NONE;
    if (!has_branch) return edge_back_t<X, false, false, true>(a, cus, s);
    if (after) return before ? edge_back_t<X, true, true, true>(a, cus, s) : edge_back_t<X, true, true, false>(a, cus, s);
    return before ? edge_back_t<X, true, false, true>(a, cus, s) : edge_back_t<X, true, false, false>(a, cus, s);
}
hipError_t launch_column_total(bool bf16, const float *part, int32_t blocks, int32_t n, void *out, hipStream_t s)
{
    const TotalArgs t{part, {out}, 1, blocks, n, 0};
    return bf16 ? total_t<Bf16>(t, s) : total_t<Fp16>(t, s);
}
hipError_t launch_edge_back(bool bf16, EdgeBackArgs a, bool has_branch, void *work, int32_t cus, hipStream_t s)
{
    if (a.n == 0) return hipSuccess;
    a.sums = 0;
    for (int q = 0; q < SUMS; ++q) a.at[q] = a.sum[q] ? a.sums++ : -1;
    const bool norms = a.before.kind != DBS_NORM_NONE || a.after.kind != DBS_NORM_NONE;
    const bool both = a.before.kind != DBS_NORM_NONE && a.after.kind != DBS_NORM_NONE;
    a.blocks = sum_blocks(has_branch, both, a.rows, a.n, cus);
    a.part = (float *)work;
    a.stat = norms && a.rows > 0 && !back_fits(has_branch, a.n) ? (BackStat *)((uint8_t *)work + part_bytes(has_branch, both, a.rows, a.n, a.sums, cus)) : nullptr;
    return bf16 ? edge_back_x<Bf16>(a, has_branch, cus, s) : edge_back_x<Fp16>(a, has_branch, cus, s);
}

hipError_t launch_dropout(bool bf16, const void *x, int64_t ldx, int32_t rows, int32_t n, const Drop &d, void *y, int64_t ldy,
                          int32_t cus, hipStream_t s)
{
    if (rows == 0 || n == 0) return hipSuccess;
    const int32_t per = (n + 7) / 8;
    const int64_t chunks = (int64_t)rows * per;
    const dim3 grid((unsigned)std::min<int64_t>((chunks + DROP_TPB - 1) / DROP_TPB, 16 * (int64_t)cus)), block(DROP_TPB);
    if (bf16) hipLaunchKernelGGL(k_dropout<Bf16>, grid, block, 0, s, (const Bf16::T *)x, ldx, rows, n, per, d, (Bf16::T *)y, ldy);
    else hipLaunchKernelGGL(k_dropout<Fp16>, grid, block, 0, s, (const Fp16::T *)x, ldx, rows, n, per, d, (Fp16::T *)y, ldy);
    return hipGetLastError();
}

}  // namespace dbs
