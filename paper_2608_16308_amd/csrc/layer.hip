// C ABI of the dense layer operators: argument checks, workspaces and the
// order of the launches.
#include <algorithm>
#include <climits>
#include <cstring>
#include <new>

#include "layer_abi.hpp"

using namespace dbs;

namespace {

constexpr size_t PART_BYTES = (size_t)128 << 20;  // sums of split tiles
bool known_act(dbs_act a) { return a >= DBS_ACT_NONE && a <= DBS_ACT_GELU_TANH; }

dbs_status check_held(const char *fn, const char *name, const dbs_held *h, int64_t rows, int64_t cols)
{
    if (rows == 0 || cols == 0) return DBS_OK;
    if (!h) return dbs_fail(DBS_ERR_ARG, "%s: %s is NULL", fn, name);
    if (h->d_values && h->d_codes) return dbs_fail(DBS_ERR_ARG, "%s: %s is given both as values and as codes", fn, name);
    if (h->d_codes) return h->d_exps ? DBS_OK : dbs_fail(DBS_ERR_ARG, "%s: %s has codes and no exponents", fn, name);
    return check_operand(fn, name, h->d_values, rows, cols, h->ld);
}
dbs_status check_keep(const char *fn, const char *name, const dbs_keep *k, int64_t rows, int64_t cols)
{
    if (!k || rows == 0 || cols == 0) return DBS_OK;
    if (k->d_values && k->d_codes) return dbs_fail(DBS_ERR_ARG, "%s: %s is asked for both as values and as codes", fn, name);
    if (k->d_codes) return k->d_exps ? DBS_OK : dbs_fail(DBS_ERR_ARG, "%s: %s has codes and no exponents", fn, name);
    return check_operand(fn, name, k->d_values, rows, cols, k->ld);
}

HeldIn held_in(const dbs_held *h) { return h ? HeldIn{h->d_values, h->ld, h->d_codes, h->d_exps} : HeldIn{}; }

SaveTo save_to(const dbs_keep *k) { return k ? SaveTo{k->d_values, k->ld, k->d_codes, k->d_exps} : SaveTo{}; }

// Whether a product gains from copies of its operands in whole 16-byte chunks
// (`bytes` of them): a copy is read and written at 4.5 TB/s, after 3 us of launch,
// and the tiles that load straight into LDS then save what the tiles through
// registers are slower by.  Those lose most where operands are stored across k
// (`across`: the backward products).  fp16, us through registers / with copies:
//   linear 1531x1111->2003 27.5 / 31.6, 2000x2001->2003 39.8 / 44.8,
//          2000x3001->2003 50.0 / 49.0, 4096x4097->4096 192 / 144
//   dx     100x1111->2003 26.6 / 25.1, 777x1111->2003 38.1 / 30.0,
//          2000x3001->2003 102 / 74, 4096x4097->4096 297 / 167
//   dw     100x1111->2003 19.1 / 22.1, 777x1111->2003 42.8 / 27.6,
//          2000x3001->2003 103 / 73, 4096x4097->4096 326 / 172
// The rates are set to put the limit between them, 600 (300 across k) TFLOP/s
// against 900.
bool copies_pay(double flops, double bytes, int copies, bool across)
{
    return flops * (1 / (across ? 300e6 : 600e6) - 1 / 900e6) > 2 * bytes / 4.5e6 + 3.0 * copies;  // (us)
}
size_t rows_bytes(int64_t rows, int64_t cols) { return up256((size_t)rows * up8(cols) * 2); }

// An operand, or its copy in whole chunks.
struct Operand {
    const void *p;
    int64_t ld;
    int32_t rows, cols;
    bool whole() const { return whole_chunks(p, ld, cols); }
};
// Copies the operands that are not in whole chunks into the workspace, if that
// pays and they fit; true if they all are then.
hipError_t make_whole(const LayerWork &w, Operand *const *ops, int n, double flops, bool across, Carve &c, size_t room,
                      hipStream_t s, bool *padded)
{
    size_t bytes = 0;
    int copies = 0;
    *padded = false;
    for (int i = 0; i < n; ++i)
        if (!ops[i]->whole()) bytes += rows_bytes(ops[i]->rows, ops[i]->cols), ++copies;
    if (!copies || !c.base || c.used + bytes > room || !copies_pay(flops, (double)bytes, copies, across)) return hipSuccess;
    for (int i = 0; i < n; ++i) {
        Operand &o = *ops[i];
        if (o.whole()) continue;
        void *to = c.take(rows_bytes(o.rows, o.cols));
        const hipError_t e = launch_align(o.p, o.ld, o.rows, o.cols, to, up8(o.cols), w.cus, s);
        if (e != hipSuccess) return e;
        o.p = to, o.ld = up8(o.cols);
    }
    *padded = true;
    return hipSuccess;
}

// What a backward pass cannot do without: dz (and du) where an activation has a
// slope or dy is not in whole chunks, with the largest of them, the values of an x
// held in 8 bits, the partial sums of db.
struct BackwardWork {
    void *dz, *du, *x;
    float *most, *sums;
    int64_t blocks;
    int64_t ldz, ldx;
    Carve c;
};
BackwardWork carve(void *mem, bool gated, bool slope, bool x_codes, bool db, int64_t t, int64_t n_in, int64_t n_out, int32_t cus)
{
    BackwardWork b{};
    b.c.base = (uint8_t *)mem;
    b.ldz = up8(n_out);
    b.ldx = up8(n_in);
    b.blocks = slope_blocks(t, n_out, cus);
    if (slope) b.dz = b.c.take((size_t)t * b.ldz * 2), b.most = (float *)b.c.take((size_t)(b.blocks + 1) * 4);
    if (gated) b.du = b.c.take((size_t)t * b.ldz * 2);
    if (x_codes) b.x = b.c.take((size_t)t * b.ldx * 2);
    if (db) b.sums = (float *)b.c.take((size_t)slope_row_blocks((int32_t)t, (int32_t)n_out, cus) * n_out * 4);
    return b;
}

}  // namespace

extern "C" {

dbs_status dbs_layer_create(void *stream, dbs_layer **out)
{
    if (!out) return dbs_fail(DBS_ERR_ARG, "dbs_layer_create: out is NULL");
    *out = nullptr;
    int dev = 0;
    hipDeviceProp_t prop;
    LAYER_TRY(hipGetDevice(&dev), "hipGetDevice");
    LAYER_TRY(hipGetDeviceProperties(&prop, dev), "hipGetDeviceProperties");
    if (std::strncmp(prop.gcnArchName, "gfx950", 6) != 0)
        return dbs_fail(DBS_ERR_DEVICE, "dbs_layer_create: this build runs on gfx950, the device is %s", prop.gcnArchName);
    dbs_layer *L = new (std::nothrow) dbs_layer();
    if (!L) return dbs_fail(DBS_ERR_ALLOC, "dbs_layer_create: host allocation");
    const size_t zeros = 256;
    hipError_t e = hipMalloc(&L->mem, zeros + PART_BYTES);
    if (e == hipSuccess) e = hipMemset(L->mem, 0, zeros);
    if (e == hipSuccess) e = hipStreamSynchronize(nullptr);  // (calls may run on streams that do not wait for this one)
    if (e == hipSuccess) e = hipDeviceGetAttribute(&L->w.cus, hipDeviceAttributeMultiprocessorCount, dev);
    if (e != hipSuccess) {
        dbs_layer_destroy(L);
        return layer_hip_fail(e, "dbs_layer_create");
    }
    L->w.zeros = L->mem;
    L->w.part = (float *)((uint8_t *)L->mem + zeros);
    L->w.part_bytes = PART_BYTES;
    L->stream = (hipStream_t)stream;
    *out = L;
    return DBS_OK;
}

void dbs_layer_destroy(dbs_layer *L)
{
    if (!L) return;
    if (L->mem) (void)hipFree(L->mem);
    delete L;
}

// x and the one or two weights of a forward product, few tokens as they are.
static dbs_status forward_operands(dbs_layer *L, const char *fn, Operand *const *ops, int n, GemmArgs &a, void *d_work,
                                   size_t work_bytes)
{
    a.pn = ops[1]->rows, a.qn = ops[0]->rows, a.kn = ops[0]->cols, a.segs = 1, a.batch = 1;
    bool padded = false;
    Carve c{(uint8_t *)d_work};
    if (a.qn > ROWS_TOKENS)
        LAYER_TRY(make_whole(L->w, ops, n, 2.0 * (n - 1) * a.qn * a.kn * a.pn, false, c, work_bytes, L->stream, &padded), fn);
    a.p_padded = a.q_padded = padded;
    a.q[0] = ops[0]->p, a.ldq[0] = ops[0]->ld;
    for (int i = 1; i < n; ++i) a.p[i - 1] = ops[i]->p, a.ldp[i - 1] = ops[i]->ld;
    return DBS_OK;
}

dbs_status dbs_forward_work(const dbs_layer *L, int gated, int32_t t, int32_t n_in, int32_t n_out, size_t *bytes)
{
    CHECK(check_call("dbs_forward_work", L, DBS_F16, t, n_in, n_out));
    if (!bytes) return dbs_fail(DBS_ERR_ARG, "dbs_forward_work: bytes is NULL");
    const int n = gated ? 2 : 1;
    const size_t x = rows_bytes(t, n_in), w = n * rows_bytes(n_out, n_in);
    *bytes = t > ROWS_TOKENS && copies_pay(2.0 * n * t * n_in * n_out, (double)std::min(x, w), 1, false) ? x + w : 0;
    return DBS_OK;
}

dbs_status dbs_linear(dbs_layer *L, dbs_dtype dt, int32_t t, int32_t n_in, int32_t n_out, const void *d_x, int64_t ldx,
                      const void *d_w, int64_t ldw, const void *d_bias, dbs_act act, const void *d_res, int64_t ldr,
                      void *d_y, int64_t ldy, const dbs_keep *pre, void *d_work, size_t work_bytes)
{
    const char *fn = "dbs_linear";
    CHECK(check_call(fn, L, dt, t, n_in, n_out));
    if (!known_act(act)) return dbs_fail(DBS_ERR_ARG, "%s: unknown activation %d", fn, (int)act);
    CHECK(check_operand(fn, "x", d_x, t, n_in, ldx));
    CHECK(check_operand(fn, "w", d_w, n_out, n_in, ldw));
    if (d_bias) CHECK(check_operand(fn, "bias", d_bias, 1, n_out, n_out));
    if (d_res) CHECK(check_operand(fn, "residual", d_res, t, n_out, ldr));
    CHECK(check_operand(fn, "y", d_y, t, n_out, ldy));
    CHECK(check_keep(fn, "pre", pre, t, n_out));
    CHECK(check_work(fn, d_work));
    GemmArgs a{};
    Operand x{d_x, ldx, t, n_in}, w{d_w, ldw, n_out, n_in}, *const ops[] = {&x, &w};
    CHECK(forward_operands(L, fn, ops, 2, a, d_work, work_bytes));
    a.y[0] = d_y, a.ldy[0] = ldy, a.bias = d_bias, a.res = d_res, a.ldr = ldr, a.act = Act::of(act);
    a.save[0] = save_to(pre);
    LAYER_TRY(launch_gemm(L->w, dt == DBS_BF16, G_LINEAR, a, L->stream), fn);
    return DBS_OK;
}

dbs_status dbs_gated(dbs_layer *L, dbs_dtype dt, int32_t t, int32_t n_in, int32_t n_out, const void *d_x, int64_t ldx,
                     const void *d_wg, int64_t ldwg, const void *d_wu, int64_t ldwu, dbs_act act, void *d_h, int64_t ldh,
                     const dbs_keep *gate, const dbs_keep *up, void *d_work, size_t work_bytes)
{
    const char *fn = "dbs_gated";
    CHECK(check_call(fn, L, dt, t, n_in, n_out));
    if (!known_act(act)) return dbs_fail(DBS_ERR_ARG, "%s: unknown activation %d", fn, (int)act);
    if ((gate == nullptr) != (up == nullptr)) return dbs_fail(DBS_ERR_ARG, "%s: gate and up are kept together", fn);
    CHECK(check_operand(fn, "x", d_x, t, n_in, ldx));
    CHECK(check_operand(fn, "w_gate", d_wg, n_out, n_in, ldwg));
    CHECK(check_operand(fn, "w_up", d_wu, n_out, n_in, ldwu));
    CHECK(check_operand(fn, "h", d_h, t, n_out, ldh));
    CHECK(check_keep(fn, "gate", gate, t, n_out));
    CHECK(check_keep(fn, "up", up, t, n_out));
    if (gate && t > 0 && n_out > 0 && (gate->d_codes == nullptr) != (up->d_codes == nullptr))
        return dbs_fail(DBS_ERR_ARG, "%s: gate and up are kept in one form", fn);
    CHECK(check_work(fn, d_work));
    GemmArgs a{};
    Operand x{d_x, ldx, t, n_in}, g{d_wg, ldwg, n_out, n_in}, u{d_wu, ldwu, n_out, n_in}, *const ops[] = {&x, &g, &u};
    CHECK(forward_operands(L, fn, ops, 3, a, d_work, work_bytes));
    a.y[0] = d_h, a.ldy[0] = ldh, a.act = Act::of(act);
    a.save[0] = save_to(gate), a.save[1] = save_to(up);
    LAYER_TRY(launch_gemm(L->w, dt == DBS_BF16, G_GATED, a, L->stream), fn);
    return DBS_OK;
}

dbs_status dbs_backward_work(const dbs_layer *L, int gated, dbs_act act, int32_t t, int32_t n_in, int32_t n_out, int x_codes,
                             int want_db, int whole, size_t *bytes)
{
    CHECK(check_call("dbs_backward_work", L, DBS_F16, t, n_in, n_out));
    if (!bytes) return dbs_fail(DBS_ERR_ARG, "dbs_backward_work: bytes is NULL");
    const int n = gated ? 2 : 1;
    *bytes = carve(nullptr, gated != 0, gated || act != DBS_ACT_NONE || !whole, x_codes != 0, !gated && want_db, t, n_in, n_out, L->w.cus).c.used;
    if (whole) return DBS_OK;
    const double flops = 2.0 * n * t * n_in * n_out;
    const size_t x = rows_bytes(t, n_in), w = rows_bytes(n_out, n_in);
    if (copies_pay(flops, (double)w, 1, true)) *bytes += n * w;
    if (!x_codes && copies_pay(flops, (double)x, 1, true)) *bytes += x;
    return DBS_OK;
}

// The products that both backward passes end in, dz (and du) given in whole
// chunks, times 1 / *scale where that is given.
static dbs_status gradients(dbs_layer *L, const char *fn, dbs_dtype dt, int32_t t, int32_t n_in, int32_t n_out, int n,
                            const void *const dz[2], int64_t ldz, bool own_dz, const float *scale, const dbs_held *x, BackwardWork &b,
                            size_t room, Operand *const *w, void *d_dx, int64_t lddx, void *const dw[2], const int64_t lddw[2])
{
    const bool bf = dt == DBS_BF16;
    const double flops = 2.0 * n * t * n_in * n_out;
    bool padded = false;
    if (d_dx) {
        LAYER_TRY(make_whole(L->w, w, n, flops, true, b.c, room, L->stream, &padded), fn);
        GemmArgs a{};
        for (int i = 0; i < n; ++i) a.p[i] = w[i]->p, a.ldp[i] = w[i]->ld, a.q[i] = dz[i], a.ldq[i] = ldz;
        a.pn = n_in, a.qn = t, a.kn = n_out, a.segs = n, a.batch = 1;
        a.y[0] = d_dx, a.ldy[0] = lddx;
        a.p_padded = padded, a.q_padded = own_dz, a.scale = scale;
        LAYER_TRY(launch_gemm(L->w, bf, G_DX, a, L->stream), fn);
    }
    if (dw[0]) {
        Operand xv{x ? x->d_values : nullptr, x ? x->ld : 0, t, n_in}, *const ops[] = {&xv};
        if (b.x) {
            LAYER_TRY(launch_unpack(bf, x->d_codes, x->d_exps, t, n_in, b.x, b.ldx, L->w.cus, L->stream), fn);
            xv.p = b.x, xv.ld = b.ldx;
            padded = true;
        } else LAYER_TRY(make_whole(L->w, ops, 1, flops, true, b.c, room, L->stream, &padded), fn);
        GemmArgs a{};
        for (int i = 0; i < n; ++i) a.q[i] = dz[i], a.ldq[i] = ldz, a.y[i] = dw[i], a.ldy[i] = lddw[i];
        a.p[0] = xv.p, a.ldp[0] = xv.ld, a.p_padded = padded, a.q_padded = own_dz, a.scale = scale;
        a.pn = n_in, a.qn = n_out, a.kn = t, a.segs = 1, a.batch = n;
        LAYER_TRY(launch_gemm(L->w, bf, G_DW, a, L->stream), fn);
    }
    return DBS_OK;
}

dbs_status dbs_linear_backward(dbs_layer *L, dbs_dtype dt, int32_t t, int32_t n_in, int32_t n_out, const void *d_dy,
                               int64_t lddy, const dbs_held *x, const void *d_w, int64_t ldw, const dbs_held *pre, dbs_act act,
                               void *d_dx, int64_t lddx, void *d_dw, int64_t lddw, void *d_db, void *d_work, size_t work_bytes)
{
    const char *fn = "dbs_linear_backward";
    CHECK(check_call(fn, L, dt, t, n_in, n_out));
    if (!known_act(act)) return dbs_fail(DBS_ERR_ARG, "%s: unknown activation %d", fn, (int)act);
    CHECK(check_operand(fn, "dy", d_dy, t, n_out, lddy));
    if (act != DBS_ACT_NONE) CHECK(check_held(fn, "pre", pre, t, n_out));
    if (d_dx) {
        CHECK(check_operand(fn, "w", d_w, n_out, n_in, ldw));
        CHECK(check_operand(fn, "dx", d_dx, t, n_in, lddx));
    }
    if (d_dw) {
        CHECK(check_held(fn, "x", x, t, n_in));
        CHECK(check_operand(fn, "dw", d_dw, n_out, n_in, lddw));
    }
    if (d_db) CHECK(check_operand(fn, "db", d_db, 1, n_out, n_out));
    // (a dy that is not in whole chunks becomes a dz that is, also without a slope;
    // one with rows too far apart for the tiles that load them is read as it is)
    const bool chunks = (uintptr_t)d_dy % 16 == 0 && (t <= 1 || lddy % 8 == 0) && n_out % 8 == 0;
    const bool slope = act != DBS_ACT_NONE || !chunks, x_codes = d_dw && x && x->d_codes;
    BackwardWork b = carve(d_work, false, slope, x_codes, d_db != nullptr, t, n_in, n_out, L->w.cus);
    CHECK(check_room(fn, b.c.used, d_work, work_bytes));
    // (ReLU passes or drops dy as it is)
    const bool range = dt == DBS_F16 && act != DBS_ACT_NONE && act != DBS_ACT_RELU && t > 0 && n_out > 0 && (d_dx || d_dw);
    if (slope || d_db) {
        SlopeArgs s{};
        s.dy = d_dy, s.lddy = lddy, s.rows = t, s.cols = n_out, s.act = Act::of(act);
        if (act != DBS_ACT_NONE) s.pre = held_in(pre);
        s.dz = b.dz, s.ldz = b.ldz, s.most = range ? b.most : nullptr;
        s.sums = d_db ? b.sums : nullptr, s.db = d_db, s.row_blocks = slope_row_blocks(t, n_out, L->w.cus);
        LAYER_TRY(launch_slope(dt == DBS_BF16, false, s, L->stream), fn);
    }
    const void *dz[2] = {slope ? b.dz : d_dy, nullptr};
    Operand w{d_w, ldw, n_out, n_in}, *const ws[] = {&w};
    void *dw[2] = {d_dw, nullptr};
    const int64_t lddws[2] = {lddw, 0};
    return gradients(L, fn, dt, t, n_in, n_out, 1, dz, slope ? b.ldz : lddy, slope, range ? b.most + b.blocks : nullptr, x, b, work_bytes, ws, d_dx, lddx, dw, lddws);
}

dbs_status dbs_gated_backward(dbs_layer *L, dbs_dtype dt, int32_t t, int32_t n_in, int32_t n_out, const void *d_dh,
                              int64_t lddh, const dbs_held *x, const void *d_wg, int64_t ldwg, const void *d_wu, int64_t ldwu,
                              const dbs_held *gate, const dbs_held *up, dbs_act act, void *d_dx, int64_t lddx, void *d_dwg,
                              int64_t lddwg, void *d_dwu, int64_t lddwu, void *d_work, size_t work_bytes)
{
    const char *fn = "dbs_gated_backward";
    CHECK(check_call(fn, L, dt, t, n_in, n_out));
    if (!known_act(act)) return dbs_fail(DBS_ERR_ARG, "%s: unknown activation %d", fn, (int)act);
    if ((d_dwg == nullptr) != (d_dwu == nullptr)) return dbs_fail(DBS_ERR_ARG, "%s: dw_gate and dw_up are taken together", fn);
    CHECK(check_operand(fn, "dh", d_dh, t, n_out, lddh));
    CHECK(check_held(fn, "gate", gate, t, n_out));
    CHECK(check_held(fn, "up", up, t, n_out));
    if (d_dx) {
        CHECK(check_operand(fn, "w_gate", d_wg, n_out, n_in, ldwg));
        CHECK(check_operand(fn, "w_up", d_wu, n_out, n_in, ldwu));
        CHECK(check_operand(fn, "dx", d_dx, t, n_in, lddx));
    }
    if (d_dwg) {
        CHECK(check_held(fn, "x", x, t, n_in));
        CHECK(check_operand(fn, "dw_gate", d_dwg, n_out, n_in, lddwg));
        CHECK(check_operand(fn, "dw_up", d_dwu, n_out, n_in, lddwu));
    }
    const bool x_codes = d_dwg && x && x->d_codes;
    BackwardWork b = carve(d_work, true, true, x_codes, false, t, n_in, n_out, L->w.cus);
    CHECK(check_room(fn, b.c.used, d_work, work_bytes));
    const bool range = dt == DBS_F16 && t > 0 && n_out > 0;
    if (t > 0) {
        SlopeArgs s{};
        s.dy = d_dh, s.lddy = lddh, s.pre = held_in(gate), s.up = held_in(up), s.rows = t, s.cols = n_out, s.act = Act::of(act);
        s.dz = b.dz, s.du = b.du, s.ldz = b.ldz, s.row_blocks = slope_row_blocks(t, n_out, L->w.cus);
        s.most = range ? b.most : nullptr;
        LAYER_TRY(launch_slope(dt == DBS_BF16, true, s, L->stream), fn);
    }
    const void *dz[2] = {b.dz, b.du};
    Operand g{d_wg, ldwg, n_out, n_in}, u{d_wu, ldwu, n_out, n_in}, *const ws[] = {&g, &u};
    void *dw[2] = {d_dwg, d_dwu};
    const int64_t lddw[2] = {lddwg, lddwu};
    return gradients(L, fn, dt, t, n_in, n_out, 2, dz, b.ldz, true, range ? b.most + b.blocks : nullptr, x, b, work_bytes, ws, d_dx, lddx, dw, lddw);
}

dbs_status dbs_pack(dbs_layer *L, dbs_dtype dt, int32_t rows, int32_t cols, const void *d_x, int64_t ldx, int8_t *d_codes,
                    uint8_t *d_exps)
{
    CHECK(check_call("dbs_pack", L, dt, rows, cols, 0));
    CHECK(check_operand("dbs_pack", "x", d_x, rows, cols, ldx));
    if (rows > 0 && cols > 0 && (!d_codes || !d_exps)) return dbs_fail(DBS_ERR_ARG, "dbs_pack: NULL output");
    LAYER_TRY(launch_pack(dt == DBS_BF16, d_x, ldx, rows, cols, d_codes, d_exps, L->w.cus, L->stream), "dbs_pack");
    return DBS_OK;
}

dbs_status dbs_unpack(dbs_layer *L, dbs_dtype dt, int32_t rows, int32_t cols, const int8_t *d_codes, const uint8_t *d_exps,
                      void *d_y, int64_t ldy)
{
    CHECK(check_call("dbs_unpack", L, dt, rows, cols, 0));
    CHECK(check_operand("dbs_unpack", "y", d_y, rows, cols, ldy));
    if (rows > 0 && cols > 0 && (!d_codes || !d_exps)) return dbs_fail(DBS_ERR_ARG, "dbs_unpack: NULL input");
    LAYER_TRY(launch_unpack(dt == DBS_BF16, d_codes, d_exps, rows, cols, d_y, ldy, L->w.cus, L->stream), "dbs_unpack");
    return DBS_OK;
}

}  // extern "C"
