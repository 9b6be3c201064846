// C ABI of the two ends of a training step: the classifier's loss and the orthogonalised update.  Checks come before any launch.
#include <stdio.h>

#include "api_check.h"
#include "train_ends.h"

namespace cac {

static const char *tile_name(const TileChoice &c)
{
    static const char *const names[] = {"64", "128", "192", "256", "32 x 128"};
    return names[c.shape];
}

// A call's buffers: the first `outputs` are written, the others are read or are workspace.  No output may share memory with another
// buffer (null and empty ones are left out).
struct Buffer {
    const void *p;
    size_t bytes;
    const char *name;
};
static int check_apart(const Buffer *b, int outputs, int all)
{
    for (int i = 0; i < outputs; ++i)
        for (int k = i + 1; k < all; ++k)
            if (b[i].p && b[k].p && b[k].bytes && share_memory(b[i].p, b[i].bytes, b[k].p, b[k].bytes))
                return fail(CAC_ERR_INVALID_ARG, "%s shares memory with %s", b[i].name, b[k].name);
    return CAC_OK;
}

static size_t bytes_of(int dtype) { return dtype == CAC_F32 ? 4 : 2; }
// from the first number of a matrix to behind its last
static size_t rows_bytes(long rows, long columns, long ld, size_t e) { return ((size_t)(rows - 1) * ld + columns) * e; }

static int make_loss_geom(const cac_loss_desc *d, LossGeom *g)
{
    if (!d) return fail(CAC_ERR_INVALID_ARG, "descriptor is NULL");
    if (d->size != sizeof(cac_loss_desc))
        return fail(CAC_ERR_INVALID_ARG, "desc.size is %u, this library expects %zu", d->size, sizeof(cac_loss_desc));
    if (d->T <= 0 || d->D <= 0 || d->V <= 0) return fail(CAC_ERR_INVALID_ARG, "T, D and V must be positive");
    if (d->dtype != CAC_F32 && d->dtype != CAC_BF16) return fail(CAC_ERR_INVALID_ARG, "unknown dtype %d", d->dtype);
    if ((d->ld_h && d->ld_h < d->D) || (d->ld_w && d->ld_w < d->D))
        return fail(CAC_ERR_INVALID_ARG, "ld_h and ld_w are 0 (dense rows) or at least D");
    // what keeps offsets inside a tile, and grids, in 32 bits
    if (d->T > 1 << 22 || d->V > 1 << 24 || d->D > 1 << 18 || d->ld_h > 1 << 20 || d->ld_w > 1 << 20)
        return fail(CAC_ERR_UNSUPPORTED, "T above 2^22, V above 2^24, D above 2^18 or a row stride above 2^20");
    g->T = d->T;
    g->D = d->D;
    g->V = d->V;
    g->ld_h = d->ld_h ? d->ld_h : d->D;
    g->ld_w = d->ld_w ? d->ld_w : d->D;
    g->dtype = d->dtype;
    g->bias = d->has_bias != 0;
    g->ignore = d->ignore_index;
    return CAC_OK;
}

static int make_muon_geom(const cac_muon_desc *d, MuonGeom *g, MuonPlan *p)
{
    if (!d) return fail(CAC_ERR_INVALID_ARG, "descriptor is NULL");
    if (d->size != sizeof(cac_muon_desc))
        return fail(CAC_ERR_INVALID_ARG, "desc.size is %u, this library expects %zu", d->size, sizeof(cac_muon_desc));
    if (d->rows <= 0 || d->cols <= 0 || d->batch <= 0) return fail(CAC_ERR_INVALID_ARG, "rows, cols and batch must be positive");
    if ((d->dtype != CAC_F32 && d->dtype != CAC_BF16) || (d->grad_dtype != CAC_F32 && d->grad_dtype != CAC_BF16))
        return fail(CAC_ERR_INVALID_ARG, "unknown dtype %d or grad_dtype %d", d->dtype, d->grad_dtype);
    if (d->steps < 1 || d->steps > 32) return fail(CAC_ERR_INVALID_ARG, "steps must be 1 to 32");
    if (d->rows > 1 << 18 || d->cols > 1 << 18 || d->batch > 65535)
        return fail(CAC_ERR_UNSUPPORTED, "rows or cols above 2^18 or batch above 65535");
    g->rows = d->rows;
    g->cols = d->cols;
    g->batch = d->batch;
    g->steps = d->steps;
    g->dtype = d->dtype;
    g->grad_dtype = d->grad_dtype;
    g->nesterov = d->nesterov != 0;
    plan_muon(*g, p);
    if (!p->fits) return fail(CAC_ERR_UNSUPPORTED, "batch of matrices too large for one grid");
    return CAC_OK;
}

} // namespace cac

using namespace cac;

extern "C" {

int cac_loss_workspace_size(const cac_loss_desc *d, int op, size_t *bytes)
{
    LossGeom g;
    int rc = make_loss_geom(d, &g);
    if (rc) return rc;
    if (op != CAC_LOSS_FWD && op != CAC_LOSS_BWD) return fail(CAC_ERR_INVALID_ARG, "unknown op %d", op);
    if (!bytes) return fail(CAC_ERR_INVALID_ARG, "bytes is NULL");
    LossPlan p;
    plan_loss(g, op == CAC_LOSS_BWD, &p);
    *bytes = p.bytes;
    return CAC_OK;
}

int cac_loss_describe_plan(const cac_loss_desc *d, int op, char *buf, size_t buf_len)
{
    LossGeom g;
    int rc = make_loss_geom(d, &g);
    if (rc) return rc;
    if (op != CAC_LOSS_FWD && op != CAC_LOSS_BWD) return fail(CAC_ERR_INVALID_ARG, "unknown op %d", op);
    if (!buf || buf_len == 0) return fail(CAC_ERR_INVALID_ARG, "buf is NULL or empty");
    LossPlan p;
    plan_loss(g, op == CAC_LOSS_BWD, &p);
    const int n = snprintf(buf, buf_len, "%s operands, weights %s, %d pieces of %ld classes, logits tile %s", p.split ? "two halves" : p.raw ? "float" : "bfloat16",
                           p.pack_w ? "packed" : "as they lie", p.pieces, p.piece, tile_name(p.z));
    if (op == CAC_LOSS_BWD && n > 0 && (size_t)n < buf_len)
        snprintf(buf + n, buf_len - n, ", dW tile %s, dH tile %s in %d slices", tile_name(p.w), tile_name(p.h), p.h.slices);
    return CAC_OK;
}

int cac_loss_fwd(const cac_loss_desc *d, const void *H, const void *W, const void *b, const int64_t *labels, float *loss, float *lse,
                 void *ws, size_t ws_bytes, void *stream)
{
    LossGeom g;
    int rc = make_loss_geom(d, &g);
    if (rc) return rc;
    if ((rc = check_ptr(H, "H")) || (rc = check_ptr(W, "W")) || (rc = check_ptr(labels, "labels")) || (rc = check_ptr(loss, "loss")) ||
        (rc = check_ptr(lse, "lse")))
        return rc;
    if (g.bias && (rc = check_ptr(b, "b"))) return rc;
    LossPlan p;
    plan_loss(g, false, &p);
    if ((rc = check_ws(p.bytes, ws, ws_bytes))) return rc;
    const size_t e = bytes_of(g.dtype);
    const Buffer buffers[] = {{loss, 4 * (size_t)g.T, "loss"}, {lse, 4 * (size_t)g.T, "lse"}, {H, rows_bytes(g.T, g.D, g.ld_h, e), "H"},
                              {W, rows_bytes(g.V, g.D, g.ld_w, e), "W"}, {g.bias ? b : nullptr, g.V * e, "b"}, {labels, 8 * (size_t)g.T, "labels"},
                              {ws, p.bytes, "the workspace"}};
    if ((rc = check_apart(buffers, 2, 7))) return rc;
    return launched(launch_loss_fwd(g, p, H, W, g.bias ? b : nullptr, labels, loss, lse, ws, (hipStream_t)stream), "cross entropy");
}

int cac_loss_bwd(const cac_loss_desc *d, const void *H, const void *W, const void *b, const int64_t *labels, const float *lse,
                 const float *gloss, void *dH, void *dW, void *db, void *ws, size_t ws_bytes, void *stream)
{
    LossGeom g;
    int rc = make_loss_geom(d, &g);
    if (rc) return rc;
    if ((rc = check_ptr(H, "H")) || (rc = check_ptr(W, "W")) || (rc = check_ptr(labels, "labels")) || (rc = check_ptr(lse, "lse")) ||
        (rc = check_ptr(gloss, "gloss")))
        return rc;
    if (g.bias && (rc = check_ptr(b, "b"))) return rc;
    if (!dH && !dW && !db) return fail(CAC_ERR_INVALID_ARG, "dH, dW and db are all NULL: nothing to compute");
    if ((dH && (rc = check_ptr(dH, "dH"))) || (dW && (rc = check_ptr(dW, "dW"))) || (db && (rc = check_ptr(db, "db")))) return rc;
    LossPlan p;
    plan_loss(g, true, &p);
    if ((rc = check_ws(p.bytes, ws, ws_bytes))) return rc;
    const size_t e = bytes_of(g.dtype);
    const bool in_place = dH == H && g.ld_h == g.D;
    const Buffer buffers[] = {{dH, g.T * g.D * e, "dH"}, {dW, g.V * g.D * e, "dW"}, {db, g.V * e, "db"},
                              {in_place ? nullptr : H, rows_bytes(g.T, g.D, g.ld_h, e), "H"}, {W, rows_bytes(g.V, g.D, g.ld_w, e), "W"},
                              {g.bias ? b : nullptr, g.V * e, "b"}, {labels, 8 * (size_t)g.T, "labels"}, {lse, 4 * (size_t)g.T, "lse"},
                              {gloss, 4 * (size_t)g.T, "gloss"}, {ws, p.bytes, "the workspace"}};
    if ((rc = check_apart(buffers, 3, 10))) return rc;
    return launched(launch_loss_bwd(g, p, H, W, g.bias ? b : nullptr, labels, lse, gloss, dH, dW, db, ws, (hipStream_t)stream),
                    "cross entropy backward");
}

int cac_muon_workspace_size(const cac_muon_desc *d, int op, size_t *bytes)
{
    MuonGeom g;
    MuonPlan p;
    int rc = make_muon_geom(d, &g, &p);
    if (rc) return rc;
    if (op != CAC_MUON_ORTHOGONALISE && op != CAC_MUON_STEP) return fail(CAC_ERR_INVALID_ARG, "unknown op %d", op);
    if (!bytes) return fail(CAC_ERR_INVALID_ARG, "bytes is NULL");
    *bytes = p.bytes;
    return CAC_OK;
}

int cac_muon_describe_plan(const cac_muon_desc *d, int op, char *buf, size_t buf_len)
{
    MuonGeom g;
    MuonPlan p;
    int rc = make_muon_geom(d, &g, &p);
    if (rc) return rc;
    if (op != CAC_MUON_ORTHOGONALISE && op != CAC_MUON_STEP) return fail(CAC_ERR_INVALID_ARG, "unknown op %d", op);
    if (!buf || buf_len == 0) return fail(CAC_ERR_INVALID_ARG, "buf is NULL or empty");
    if (p.narrow)
        snprintf(buf, buf_len, "narrow: %d workgroups of %d columns, %d launches", p.np.slices, p.np.width, p.np.slices == 1 ? 1 : g.steps + 1);
    else
        snprintf(buf, buf_len, "%s, square products of %ld: tile %s in %d slices, then %s; tile %s", p.tall ? "X^T X" : "X X^T", p.r, tile_name(p.gram),
                 p.gram.slices, tile_name(p.poly), tile_name(p.apply));
    return CAC_OK;
}

int cac_orthogonalise(const cac_muon_desc *d, const void *G, void *O, void *ws, size_t ws_bytes, void *stream)
{
    MuonGeom g;
    MuonPlan p;
    int rc = make_muon_geom(d, &g, &p);
    if (rc) return rc;
    if ((rc = check_ptr(G, "G")) || (rc = check_ptr(O, "O"))) return rc;
    if ((rc = check_ws(p.bytes, ws, ws_bytes))) return rc;
    const size_t n = (size_t)g.batch * g.rows * g.cols;
    const bool in_place = O == G && g.dtype == g.grad_dtype;
    const Buffer buffers[] = {{O, n * bytes_of(g.dtype), "O"}, {in_place ? nullptr : G, n * bytes_of(g.grad_dtype), "G"}, {ws, p.bytes, "the workspace"}};
    if ((rc = check_apart(buffers, 1, 3))) return rc;
    return launched(launch_muon(g, p, G, nullptr, nullptr, O, 0.f, 0.f, 0.f, ws, (hipStream_t)stream), "orthogonalise");
}

int cac_muon_step(const cac_muon_desc *d, const void *G, float *M, void *W, float momentum, float keep, float lr, void *ws, size_t ws_bytes,
                  void *stream)
{
    MuonGeom g;
    MuonPlan p;
    int rc = make_muon_geom(d, &g, &p);
    if (rc) return rc;
    if ((rc = check_ptr(G, "G")) || (rc = check_ptr(M, "M")) || (rc = check_ptr(W, "W"))) return rc;
    if ((rc = check_ws(p.bytes, ws, ws_bytes))) return rc;
    const size_t n = (size_t)g.batch * g.rows * g.cols;
    const Buffer buffers[] = {{M, n * 4, "M"}, {W, n * bytes_of(g.dtype), "W"}, {G, n * bytes_of(g.grad_dtype), "G"}, {ws, p.bytes, "the workspace"}};
    if ((rc = check_apart(buffers, 2, 4))) return rc;
    return launched(launch_muon(g, p, G, M, W, nullptr, momentum, keep, lr, ws, (hipStream_t)stream), "momentum and orthogonalised update");
}

} // extern "C"
