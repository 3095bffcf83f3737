// C ABI of the norms, joins and dropout: argument checks and launches.
#include <cmath>

#include "layer_abi.hpp"
#include "norm.hpp"

using namespace dbs;

namespace {

dbs_status check_norm(const char *fn, const char *name, const dbs_norm_desc *d, int64_t n, NormOf &out)
{
    out = NormOf{};
    if (!d || d->kind == DBS_NORM_NONE) return DBS_OK;
    if (d->kind != DBS_NORM_RMS && d->kind != DBS_NORM_LAYER) return dbs_fail(DBS_ERR_ARG, "%s: unknown kind %d of %s", fn, (int)d->kind, name);
    if (!(d->eps >= 0.f) || !std::isfinite(d->eps)) return dbs_fail(DBS_ERR_ARG, "%s: eps of %s must be a finite number, at least 0", fn, name);
    if (d->d_weight) CHECK(check_operand(fn, "a norm's weight", d->d_weight, 1, n, n));
    if (d->d_bias) CHECK(check_operand(fn, "a norm's bias", d->d_bias, 1, n, n));
    out = NormOf{(int32_t)d->kind, d->eps, d->d_weight, d->d_bias};
    return DBS_OK;
}

dbs_status check_drop(const char *fn, const dbs_drop_desc *d, Drop &out)
{
    out = Drop{0, 1.f, 0, 0, nullptr};
    if (!d) return DBS_OK;
    if (!(d->p >= 0.0 && d->p <= 1.0)) return dbs_fail(DBS_ERR_ARG, "%s: p must be between 0 and 1", fn);
    if ((uintptr_t)d->d_rng % 8) return dbs_fail(DBS_ERR_ARG, "%s: the seed and offset in device memory are not aligned to 8 bytes", fn);
    const uint32_t t = (uint32_t)std::floor(d->p * 65536.0 + 0.5);
    out = Drop{t, t < 65536u ? (float)(65536.0 / (65536.0 - t)) : 0.f, d->seed, d->offset, d->d_rng};
    return DBS_OK;
}

// A gate [n] (ldg 0) or [rows, n].
dbs_status check_gate(const char *fn, const void *gate, int64_t rows, int64_t n, int64_t ldg)
{
    if (!gate) return DBS_OK;
    return check_operand(fn, "gate", gate, ldg == 0 ? 1 : rows, n, ldg == 0 ? n : ldg);
}

dbs_status check_blocks(const char *fn, const dbs_blocks8 *b, int64_t rows, int64_t n)
{
    if (!b || rows == 0 || n == 0) return DBS_OK;
    if (!b->d_codes || !b->d_exps) return dbs_fail(DBS_ERR_ARG, "%s: blocks without codes or exponents", fn);
    if ((uintptr_t)b->d_codes % 16 || (uintptr_t)b->d_exps % 4)
        return dbs_fail(DBS_ERR_ARG, "%s: codes must be aligned to 16 bytes, exponents to 4", fn);
    return DBS_OK;
}

}  // namespace

extern "C" {

dbs_status dbs_norm(dbs_layer *L, dbs_dtype dt, int32_t rows, int32_t n, const void *d_x, int64_t ldx, const dbs_norm_desc *norm,
                    void *d_y, int64_t ldy, const dbs_blocks8 *y8)
{
    const char *fn = "dbs_norm";
    CHECK(check_call(fn, L, dt, rows, n, 0));
    CHECK(check_operand(fn, "x", d_x, rows, n, ldx));
    if (!norm || norm->kind == DBS_NORM_NONE) return dbs_fail(DBS_ERR_ARG, "%s: no norm is given", fn);
    if ((d_y == nullptr) == (y8 == nullptr) && rows > 0 && n > 0) return dbs_fail(DBS_ERR_ARG, "%s: y is given in one form", fn);
    if (!y8) CHECK(check_operand(fn, "y", d_y, rows, n, ldy));
    CHECK(check_blocks(fn, y8, rows, n));
    EdgeArgs a{};
    CHECK(check_norm(fn, "norm", norm, n, a.before));
    a.res = d_x, a.ldr = ldx, a.scale = 1.f, a.rows = rows, a.n = n;
    if (y8) a.codes = (uint8_t *)y8->d_codes, a.exps = y8->d_exps;
    else a.h = d_y, a.ldh = ldy;
    LAYER_TRY(launch_edge(dt == DBS_BF16, a, L->w.cus, L->stream), fn);
    return DBS_OK;
}

dbs_status dbs_join(dbs_layer *L, dbs_dtype dt, int32_t rows, int32_t n, const void *d_branch, int64_t ldb, const void *d_residual,
                    int64_t ldr, const dbs_norm_desc *after, const dbs_norm_desc *before, const void *d_gate, int64_t ldg, float scale,
                    const dbs_drop_desc *drop, void *d_stream, int64_t lds, void *d_h, int64_t ldh, const dbs_blocks8 *h8)
{
    const char *fn = "dbs_join";
    CHECK(check_call(fn, L, dt, rows, n, 0));
    CHECK(check_operand(fn, "branch", d_branch, rows, n, ldb));
    CHECK(check_operand(fn, "residual", d_residual, rows, n, ldr));
    CHECK(check_operand(fn, "stream", d_stream, rows, n, lds));
    CHECK(check_gate(fn, d_gate, rows, n, ldg));
    EdgeArgs a{};
    CHECK(check_norm(fn, "after", after, n, a.after));
    CHECK(check_norm(fn, "before", before, n, a.before));
    CHECK(check_drop(fn, drop, a.drop));
    if (a.before.kind != DBS_NORM_NONE) {
        if ((d_h == nullptr) == (h8 == nullptr) && rows > 0 && n > 0) return dbs_fail(DBS_ERR_ARG, "%s: h is given in one form", fn);
        if (!h8) CHECK(check_operand(fn, "h", d_h, rows, n, ldh));
        CHECK(check_blocks(fn, h8, rows, n));
        if (h8) a.codes = (uint8_t *)h8->d_codes, a.exps = h8->d_exps;
        else a.h = d_h, a.ldh = ldh;
    } else if (d_h || h8) return dbs_fail(DBS_ERR_ARG, "%s: h without a norm", fn);
    a.branch = d_branch, a.ldb = ldb, a.res = d_residual, a.ldr = ldr, a.gate = d_gate, a.ldg = ldg, a.scale = scale;
    a.stream = d_stream, a.lds = lds, a.rows = rows, a.n = n;
    LAYER_TRY(launch_edge(dt == DBS_BF16, a, L->w.cus, L->stream), fn);
    return DBS_OK;
}

dbs_status dbs_edge_work(const dbs_layer *L, int32_t rows, int32_t n, int sums, size_t *bytes)
{
    CHECK(check_call("dbs_edge_work", L, DBS_F16, rows, n, 0));
    if (!bytes) return dbs_fail(DBS_ERR_ARG, "dbs_edge_work: bytes is NULL");
    if (sums < 0 || sums > SUMS) return dbs_fail(DBS_ERR_ARG, "dbs_edge_work: %d sums", sums);
    *bytes = edge_back_work(rows, n, sums, L->w.cus);
    return DBS_OK;
}

dbs_status dbs_norm_backward(dbs_layer *L, dbs_dtype dt, int32_t rows, int32_t n, const void *d_dy, int64_t lddy, const void *d_x,
                             int64_t ldx, const dbs_norm_desc *norm, const void *d_add, int64_t ldadd, void *d_dx, int64_t lddx,
                             void *d_dweight, void *d_dbias, void *d_work, size_t work_bytes)
{
    const char *fn = "dbs_norm_backward";
    CHECK(check_call(fn, L, dt, rows, n, 0));
    if (!norm || norm->kind == DBS_NORM_NONE) return dbs_fail(DBS_ERR_ARG, "%s: no norm is given", fn);
    CHECK(check_operand(fn, "dy", d_dy, rows, n, lddy));
    CHECK(check_operand(fn, "x", d_x, rows, n, ldx));
    if (d_add) CHECK(check_operand(fn, "add", d_add, rows, n, ldadd));
    if (d_dx) CHECK(check_operand(fn, "dx", d_dx, rows, n, lddx));
    if (d_dweight) CHECK(check_operand(fn, "dweight", d_dweight, 1, n, n));
    if (d_dbias) CHECK(check_operand(fn, "dbias", d_dbias, 1, n, n));
    EdgeBackArgs a{};
    CHECK(check_norm(fn, "norm", norm, n, a.before));
    CHECK(check_room(fn, edge_back_work(rows, n, (d_dweight != nullptr) + (d_dbias != nullptr), L->w.cus), d_work, work_bytes));
    a.ds = d_add, a.ldds = ldadd, a.dh = d_dy, a.lddh = lddy, a.stream = d_x, a.lds = ldx, a.scale = 1.f, a.drop.scale = 1.f;
    a.dres = d_dx, a.lddr = lddx, a.sum[SUM_BEFORE_W] = d_dweight, a.sum[SUM_BEFORE_B] = d_dbias, a.rows = rows, a.n = n;
    LAYER_TRY(launch_edge_back(dt == DBS_BF16, a, false, d_work, L->w.cus, L->stream), fn);
    return DBS_OK;
}

dbs_status dbs_join_backward(dbs_layer *L, dbs_dtype dt, int32_t rows, int32_t n, const void *d_dstream, int64_t ldds,
                             const void *d_dh, int64_t lddh, const void *d_branch, int64_t ldb, const void *d_stream, int64_t lds,
                             const dbs_norm_desc *after, const dbs_norm_desc *before, const void *d_gate, int64_t ldg, float scale,
                             const dbs_drop_desc *drop, void *d_dresidual, int64_t lddr, void *d_dbranch, int64_t lddb, void *d_dgate,
                             int64_t lddg, void *d_dafter_weight, void *d_dafter_bias, void *d_dbefore_weight, void *d_dbefore_bias,
                             void *d_work, size_t work_bytes)
{
    const char *fn = "dbs_join_backward";
    CHECK(check_call(fn, L, dt, rows, n, 0));
    EdgeBackArgs a{};
    CHECK(check_norm(fn, "after", after, n, a.after));
    CHECK(check_norm(fn, "before", before, n, a.before));
    CHECK(check_drop(fn, drop, a.drop));
    CHECK(check_gate(fn, d_gate, rows, n, ldg));
    if (d_dstream) CHECK(check_operand(fn, "dstream", d_dstream, rows, n, ldds));
    else if (a.before.kind == DBS_NORM_NONE && rows > 0 && n > 0) return dbs_fail(DBS_ERR_ARG, "%s: no gradient is given", fn);
    if (a.before.kind != DBS_NORM_NONE) {
        CHECK(check_operand(fn, "dh", d_dh, rows, n, lddh));
        CHECK(check_operand(fn, "stream", d_stream, rows, n, lds));
    } else if (d_dh) return dbs_fail(DBS_ERR_ARG, "%s: dh without a norm", fn);
    // (the kernels read a branch that they get: one that is not needed is neither checked nor handed on)
    const bool reads_branch = a.after.kind != DBS_NORM_NONE || d_gate;
    if (reads_branch) CHECK(check_operand(fn, "branch", d_branch, rows, n, ldb));
    if (d_dresidual) CHECK(check_operand(fn, "dresidual", d_dresidual, rows, n, lddr));
    if (d_dbranch) CHECK(check_operand(fn, "dbranch", d_dbranch, rows, n, lddb));
    if (d_dgate && !d_gate) return dbs_fail(DBS_ERR_ARG, "%s: dgate without a gate", fn);
    if (d_dgate) CHECK(check_operand(fn, "dgate", d_dgate, ldg == 0 ? 1 : rows, n, ldg == 0 ? n : lddg));
    if ((d_dafter_weight || d_dafter_bias) && a.after.kind == DBS_NORM_NONE) return dbs_fail(DBS_ERR_ARG, "%s: gradients of no norm after", fn);
    if ((d_dbefore_weight || d_dbefore_bias) && a.before.kind == DBS_NORM_NONE) return dbs_fail(DBS_ERR_ARG, "%s: gradients of no norm before", fn);
    void *const vectors[] = {d_dafter_weight, d_dafter_bias, d_dbefore_weight, d_dbefore_bias};
    for (void *v : vectors)
        if (v) CHECK(check_operand(fn, "a gradient of a norm", v, 1, n, n));
    a.sum[SUM_BEFORE_W] = d_dbefore_weight, a.sum[SUM_BEFORE_B] = d_dbefore_bias;
    a.sum[SUM_AFTER_W] = d_dafter_weight, a.sum[SUM_AFTER_B] = d_dafter_bias;
    if (ldg == 0) a.sum[SUM_GATE] = d_dgate;
    else a.dgate = d_dgate, a.lddg = lddg;
    int sums = 0;
    for (void *v : a.sum) sums += v != nullptr;
    CHECK(check_room(fn, edge_back_work(rows, n, sums, L->w.cus), d_work, work_bytes));
    a.ds = d_dstream, a.ldds = ldds, a.dh = d_dh, a.lddh = lddh, a.branch = reads_branch ? d_branch : nullptr, a.ldb = ldb, a.stream = d_stream, a.lds = lds;
    a.gate = d_gate, a.ldg = ldg, a.scale = scale, a.dres = d_dresidual, a.lddr = lddr, a.dbranch = d_dbranch, a.lddb = lddb;
    a.rows = rows, a.n = n;
    LAYER_TRY(launch_edge_back(dt == DBS_BF16, a, true, d_work, L->w.cus, L->stream), fn);
    return DBS_OK;
}

dbs_status dbs_dropout(dbs_layer *L, dbs_dtype dt, int32_t rows, int32_t n, const void *d_x, int64_t ldx, const dbs_drop_desc *drop,
                       void *d_y, int64_t ldy)
{
    const char *fn = "dbs_dropout";
    CHECK(check_call(fn, L, dt, rows, n, 0));
    if (!drop) return dbs_fail(DBS_ERR_ARG, "%s: drop is NULL", fn);
    CHECK(check_operand(fn, "x", d_x, rows, n, ldx));
    CHECK(check_operand(fn, "y", d_y, rows, n, ldy));
    Drop d;
    CHECK(check_drop(fn, drop, d));
    LAYER_TRY(launch_dropout(dt == DBS_BF16, d_x, ldx, rows, n, d, d_y, ldy, L->w.cus, L->stream), fn);
    return DBS_OK;
}

}  // extern "C"
