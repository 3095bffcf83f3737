// C ABI of the blocks of 8-bit floating point and their products.
#include "float8.hpp"
#include "layer_abi.hpp"
#include "norm.hpp"

using namespace dbs;

namespace {

constexpr int32_t MAX_SUM = 1 << 24;  // elements of a product's sum: 256 rows of a tile within 32-bit offsets

dbs_status check_blocks(const char *fn, const char *name, const dbs_blocks8 *b, int64_t rows, int64_t cols)
{
    if (rows == 0 || cols == 0) return DBS_OK;
    if (!b || !b->d_codes || !b->d_exps) return dbs_fail(DBS_ERR_ARG, "%s: %s has no codes or no exponents", fn, name);
    if ((uintptr_t)b->d_codes % 16 || (uintptr_t)b->d_exps % 4)
        return dbs_fail(DBS_ERR_ARG, "%s: codes of %s must be aligned to 16 bytes, exponents to 4", fn, name);
    return DBS_OK;
}
Blocks blocks_of(const dbs_blocks8 *b, int64_t cols, bool tile)
{
    if (!b) return Blocks{};
    return Blocks{(uint8_t *)b->d_codes, b->d_exps, e8_ld(cols), e8_ldexp(cols), tile ? 7 : 0};
}
// Room for a matrix in blocks.
Blocks take_blocks(Carve &c, int64_t rows, int64_t cols, bool tile)
{
    Blocks b{nullptr, nullptr, e8_ld(cols), e8_ldexp(cols), tile ? 7 : 0};
    b.codes = (uint8_t *)c.take((size_t)rows * b.ld);
    b.exps = (uint8_t *)c.take((size_t)(tile ? e8_blocks(rows) : rows) * b.lde);
    return b;
}

// What linear8's gradients are made from.
struct Back8 {
    Blocks dy, dyt, xt, wt;
    float *sums;
    size_t used;
};
Back8 carve_back(void *mem, int64_t t, int64_t n_in, int64_t n_out, bool dx, bool dw, bool db)
{
    Back8 b{};
    Carve c{(uint8_t *)mem};
    if (dx) b.dy = take_blocks(c, t, n_out, false), b.wt = take_blocks(c, n_in, n_out, true);
    if (dw) b.dyt = take_blocks(c, n_out, t, false), b.xt = take_blocks(c, n_in, t, false);
    if (db) b.sums = (float *)c.take((size_t)e8_blocks(t) * n_out * 4);
    b.used = c.used;
    return b;
}

}  // namespace

extern "C" {

dbs_status dbs_pack8(dbs_layer *L, dbs_dtype dt, int32_t rows, int32_t cols, const void *d_x, int64_t ldx, int tile, int across,
                     const dbs_blocks8 *out)
{
    const char *fn = "dbs_pack8";
    CHECK(check_call(fn, L, dt, rows, cols, 0));
    CHECK(check_operand(fn, "x", d_x, rows, cols, ldx));
    CHECK(check_blocks(fn, "the result", out, rows, cols));
    Pack8Args a{};
    a.x = d_x, a.ldx = ldx, a.rows = rows, a.cols = cols, a.tile = tile != 0;
    (across ? a.turned : a.to) = blocks_of(out, across ? rows : cols, tile != 0);
    LAYER_TRY(launch_pack8(dt == DBS_BF16, a, L->w.cus, L->stream), fn);
    return DBS_OK;
}

dbs_status dbs_unpack8(dbs_layer *L, dbs_dtype dt, int32_t rows, int32_t cols, int tile, const dbs_blocks8 *x, void *d_y, int64_t ldy)
{
    const char *fn = "dbs_unpack8";
    CHECK(check_call(fn, L, dt, rows, cols, 0));
    CHECK(check_blocks(fn, "x", x, rows, cols));
    CHECK(check_operand(fn, "y", d_y, rows, cols, ldy));
    LAYER_TRY(launch_unpack8(dt == DBS_BF16, blocks_of(x, cols, tile != 0), rows, cols, d_y, ldy, L->w.cus, L->stream), fn);
    return DBS_OK;
}

dbs_status dbs_linear8_work(const dbs_layer *L, int32_t t, int32_t n_in, int32_t n_out, size_t *bytes)
{
    CHECK(check_call("dbs_linear8_work", L, DBS_F16, t, n_in, n_out));
    if (!bytes) return dbs_fail(DBS_ERR_ARG, "dbs_linear8_work: bytes is NULL");
    Carve c{nullptr};
    if (!rows8_pack(t, n_in)) take_blocks(c, t, n_in, false);
    *bytes = c.used;
    return DBS_OK;
}

dbs_status dbs_linear8(dbs_layer *L, dbs_dtype dt, int32_t t, int32_t n_in, int32_t n_out, const void *d_x, int64_t ldx,
                       const dbs_blocks8 *x8, const dbs_blocks8 *w8, const void *d_bias, const void *d_res, int64_t ldr, void *d_y,
                       int64_t ldy, void *d_work, size_t work_bytes)
{
    const char *fn = "dbs_linear8";
    CHECK(check_call(fn, L, dt, t, n_in, n_out));
    if (n_in > MAX_SUM) return dbs_fail(DBS_ERR_UNSUPPORTED, "%s: n_in above 2^24", fn);
    if (x8) CHECK(check_blocks(fn, "x", x8, t, n_in));
    else CHECK(check_operand(fn, "x", d_x, t, n_in, ldx));
    CHECK(check_blocks(fn, "w", w8, n_out, n_in));
    if (d_bias) CHECK(check_operand(fn, "bias", d_bias, 1, n_out, n_out));
    if (d_res) CHECK(check_operand(fn, "residual", d_res, t, n_out, ldr));
    CHECK(check_operand(fn, "y", d_y, t, n_out, ldy));
    Mul8Args m{};
    m.q = blocks_of(x8, n_in, false);
    const bool few = t <= ROWS8_TOKENS, pack = !x8 && few && rows8_pack(t, n_in);
    if (!x8 && !pack) {
        Carve c{(uint8_t *)d_work};
        m.q = take_blocks(c, t, n_in, false);
        CHECK(check_room(fn, c.used, d_work, work_bytes));
        Pack8Args a{};
        a.x = d_x, a.ldx = ldx, a.rows = t, a.cols = n_in, a.to = m.q;
        LAYER_TRY(launch_pack8(dt == DBS_BF16, a, L->w.cus, L->stream), fn);
    }
    m.p = blocks_of(w8, n_in, true);
    m.pn = n_out, m.qn = t, m.kn = n_in, m.bias = d_bias, m.res = d_res, m.ldr = ldr, m.y = d_y, m.ldy = ldy;
    if (few) LAYER_TRY(launch_rows8(L->w, dt == DBS_BF16, m, pack ? d_x : nullptr, ldx, L->stream), fn);
    else LAYER_TRY(launch_mul8(L->w, dt == DBS_BF16, m, L->stream), fn);
    return DBS_OK;
}

dbs_status dbs_linear8_backward_work(const dbs_layer *L, int32_t t, int32_t n_in, int32_t n_out, int want_dx, int want_dw, int want_db,
                                     size_t *bytes)
{
    CHECK(check_call("dbs_linear8_backward_work", L, DBS_F16, t, n_in, n_out));
    if (!bytes) return dbs_fail(DBS_ERR_ARG, "dbs_linear8_backward_work: bytes is NULL");
    *bytes = carve_back(nullptr, t, n_in, n_out, want_dx, want_dw, want_db).used;
    return DBS_OK;
}

dbs_status dbs_linear8_backward(dbs_layer *L, dbs_dtype dt, int32_t t, int32_t n_in, int32_t n_out, const void *d_dy, int64_t lddy,
                                const void *d_x, int64_t ldx, const dbs_blocks8 *x8, const dbs_blocks8 *w8, void *d_dx, int64_t lddx,
                                void *d_dw, int64_t lddw, void *d_db, void *d_work, size_t work_bytes)
{
    const char *fn = "dbs_linear8_backward";
    CHECK(check_call(fn, L, dt, t, n_in, n_out));
    if (t > MAX_SUM || n_out > MAX_SUM) return dbs_fail(DBS_ERR_UNSUPPORTED, "%s: tokens or n_out above 2^24", fn);
    CHECK(check_operand(fn, "dy", d_dy, t, n_out, lddy));
    if (d_dx) {
        CHECK(check_blocks(fn, "w", w8, n_out, n_in));
        CHECK(check_operand(fn, "dx", d_dx, t, n_in, lddx));
    }
    if (d_dw) {
        if (x8) CHECK(check_blocks(fn, "x", x8, t, n_in));
        else CHECK(check_operand(fn, "x", d_x, t, n_in, ldx));
        CHECK(check_operand(fn, "dw", d_dw, n_out, n_in, lddw));
    }
    if (d_db) CHECK(check_operand(fn, "db", d_db, 1, n_out, n_out));
    const Back8 b = carve_back(d_work, t, n_in, n_out, d_dx != nullptr, d_dw != nullptr, d_db != nullptr);
    CHECK(check_room(fn, b.used, d_work, work_bytes));
    const bool bf = dt == DBS_BF16;
    // dy is read once for all that is made of it
    Pack8Args a{};
    a.x = d_dy, a.ldx = lddy, a.rows = t, a.cols = n_out, a.to = b.dy, a.turned = b.dyt, a.sums = b.sums;
    if (a.to.codes || a.turned.codes || a.sums) LAYER_TRY(launch_pack8(bf, a, L->w.cus, L->stream), fn);
    if (d_db) LAYER_TRY(launch_column_total(bf, b.sums, (int32_t)e8_blocks(t), n_out, d_db, L->stream), fn);
    Mul8Args m{};
    if (d_dx) {
        LAYER_TRY(launch_turn8(blocks_of(w8, n_in, true), n_out, n_in, b.wt, L->stream), fn);
        m.p = b.wt, m.q = b.dy, m.pn = n_in, m.qn = t, m.kn = n_out, m.y = d_dx, m.ldy = lddx;
        LAYER_TRY(launch_mul8(L->w, bf, m, L->stream), fn);
    }
    if (d_dw) {
        Pack8Args x{};
        x.x = d_x, x.ldx = ldx, x.from = blocks_of(x8, n_in, false), x.rows = t, x.cols = n_in, x.turned = b.xt;
        LAYER_TRY(launch_pack8(bf, x, L->w.cus, L->stream), fn);
        m.p = b.xt, m.q = b.dyt, m.pn = n_in, m.qn = n_out, m.kn = t, m.y = d_dw, m.ldy = lddw;
        LAYER_TRY(launch_mul8(L->w, bf, m, L->stream), fn);
    }
    return DBS_OK;
}

}  // extern "C"
