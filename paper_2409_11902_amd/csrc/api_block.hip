// C ABI of the residual block: the dense layer with its ending, dropout, and the norms between blocks.  Checks come before any launch.
#include <math.h>
#include <stdio.h>

#include "api_check.h"
#include "block.h"

namespace cac {

static const long kMaxRow = 1L << 20; // elements from a row to the next

static int check_dtype(int dtype)
{
    if (dtype != CAC_F32 && dtype != CAC_BF16) return fail(CAC_ERR_INVALID_ARG, "unknown dtype %d", dtype);
    return CAC_OK;
}
static int check_size(const void *d, uint32_t size, size_t expected)
{
    (void)d;
    if (size != expected) return fail(CAC_ERR_INVALID_ARG, "desc.size is %u, this library expects %zu", size, expected);
    return CAC_OK;
}
static int check_stride(long ld, long columns, const char *name)
{
    if (ld && ld < columns) return fail(CAC_ERR_INVALID_ARG, "%s is 0 (dense rows) or at least a row's length", name);
    if (ld > kMaxRow) return fail(CAC_ERR_UNSUPPORTED, "%s above 2^20", name);
    return CAC_OK;
}
// what is dropped: the probability in sixteenths of a bit's range, and the inverse of what is left
static int make_drop(float p, uint32_t site, float alpha, const uint64_t *rng, Drop *d)
{
    if (!(p >= 0.f && p <= 1.f)) return fail(CAC_ERR_INVALID_ARG, "drop_p is not in [0, 1]");
    if (site >= 1u << 24) return fail(CAC_ERR_INVALID_ARG, "site is 2^24 or more");
    if (!isfinite(alpha)) return fail(CAC_ERR_INVALID_ARG, "alpha is not finite");
    d->limit = (uint32_t)floor((double)p * 65536.0 + 0.5);
    d->site = site;
    d->scale = d->limit == 65536 ? 0.f : (float)(65536.0 / (65536 - (int)d->limit));
    if (!isfinite(alpha * d->scale)) return fail(CAC_ERR_INVALID_ARG, "alpha over the probability of being kept is not finite"); // (a kept zero would come out as NaN)
    d->rng = rng;
    return CAC_OK;
}
static int check_rng(const Drop &d, const void *rng) { return d.limit ? check_ptr(rng, "rng") : CAC_OK; }

static int make_linear(const cac_linear_desc *d, bool backward, LinearGeom *g, LinearPlan *p, Drop *drop)
{
    if (!d) return fail(CAC_ERR_INVALID_ARG, "descriptor is NULL");
    int rc = check_size(d, d->size, sizeof *d);
    if (rc) return rc;
    if (d->T <= 0 || d->D <= 0 || d->N <= 0) return fail(CAC_ERR_INVALID_ARG, "T, D and N must be positive");
    if ((rc = check_dtype(d->dtype))) return rc;
    if (d->act < CAC_ACT_NONE || d->act > CAC_ACT_SILU) return fail(CAC_ERR_INVALID_ARG, "unknown act %d", d->act);
    // what keeps offsets inside a tile, and grids, in 32 bits
    if (d->T > 1 << 22 || d->D > 1 << 18 || d->N > 1 << 18) return fail(CAC_ERR_UNSUPPORTED, "T above 2^22, D or N above 2^18");
    if ((rc = check_stride(d->ld_x, d->D, "ld_x")) || (rc = check_stride(d->ld_w, d->D, "ld_w")) || (rc = check_stride(d->ld_r, d->N, "ld_r"))) return rc;
    if ((rc = make_drop(d->drop_p, d->site, d->alpha, nullptr, drop))) return rc;
    g->T = d->T;
    g->D = d->D;
    g->N = d->N;
    g->ld_x = d->ld_x ? d->ld_x : d->D;
    g->ld_w = d->ld_w ? d->ld_w : d->D;
    g->ld_r = d->ld_r ? d->ld_r : d->N;
    g->dtype = d->dtype;
    g->act = d->act;
    g->bias = d->has_bias != 0;
    g->alpha = d->alpha;
    g->drops = drop->limit != 0;
    if (!plan_linear(*g, backward, p)) return fail(CAC_ERR_UNSUPPORTED, "a product of T, D and N is too large for one grid");
    return CAC_OK;
}

static int make_norm(const cac_block_norm_desc *d, bool backward, NormGeom *g, NormPlan *p, Drop *drop)
{
    if (!d) return fail(CAC_ERR_INVALID_ARG, "descriptor is NULL");
    int rc = check_size(d, d->size, sizeof *d);
    if (rc) return rc;
    if (d->T <= 0 || d->D <= 0) return fail(CAC_ERR_INVALID_ARG, "T and D must be positive");
    if ((rc = check_dtype(d->dtype))) return rc;
    if (d->post < CAC_NORM_NONE || d->post > CAC_NORM_LAYER || d->pre < CAC_NORM_NONE || d->pre > CAC_NORM_LAYER)
        return fail(CAC_ERR_INVALID_ARG, "unknown norm %d or %d", d->post, d->pre);
    if (d->gate_rows < 0) return fail(CAC_ERR_INVALID_ARG, "gate_rows is negative");
    if (!(d->eps_post >= 0.f && d->eps_post < INFINITY) || !(d->eps_pre >= 0.f && d->eps_pre < INFINITY))
        return fail(CAC_ERR_INVALID_ARG, "eps_post and eps_pre are finite and not negative");
    if (d->D > 1 << 14 || d->T > 1 << 28) return fail(CAC_ERR_UNSUPPORTED, "D above 2^14 or T above 2^28");
    if ((rc = check_stride(d->ld_f, d->D, "ld_f")) || (rc = check_stride(d->ld_r, d->D, "ld_r"))) return rc;
    if ((rc = make_drop(d->drop_p, d->site, d->alpha, nullptr, drop))) return rc;
    g->T = d->T;
    g->D = d->D;
    g->ld_f = d->ld_f ? d->ld_f : d->D;
    g->ld_r = d->ld_r ? d->ld_r : d->D;
    g->dtype = d->dtype;
    g->post = d->post;
    g->pre = d->pre;
    g->gate_rows = d->gate_rows < d->T ? d->gate_rows : d->T;
    g->eps_post = d->eps_post;
    g->eps_pre = d->eps_pre;
    g->alpha = d->alpha;
    plan_norm(*g, backward, p);
    return CAC_OK;
}

// null or well aligned
static int check_optional(const void *p, const char *name) { return p ? check_ptr(p, name) : CAC_OK; }
static int check_absent(const void *p, const char *name, const char *why)
{
    return p ? fail(CAC_ERR_INVALID_ARG, "%s is given, but %s", name, why) : CAC_OK;
}

} // namespace cac

using namespace cac;

extern "C" {

int cac_linear_workspace_size(const cac_linear_desc *d, int op, size_t *bytes)
{
    LinearGeom g;
    LinearPlan p;
    Drop drop;
    if (op != CAC_LINEAR_FWD && op != CAC_LINEAR_BWD) return fail(CAC_ERR_INVALID_ARG, "unknown op %d", op);
    int rc = make_linear(d, op == CAC_LINEAR_BWD, &g, &p, &drop);
    if (rc) return rc;
    if (!bytes) return fail(CAC_ERR_INVALID_ARG, "bytes is NULL");
    *bytes = p.bytes;
    return CAC_OK;
}

int cac_linear_describe_plan(const cac_linear_desc *d, int op, char *buf, size_t buf_len)
{
    static const char *const kTiles[] = {"64", "128", "192", "256", "32 x 128"};
    LinearGeom g;
    LinearPlan p;
    Drop drop;
    if (op != CAC_LINEAR_FWD && op != CAC_LINEAR_BWD) return fail(CAC_ERR_INVALID_ARG, "unknown op %d", op);
    int rc = make_linear(d, op == CAC_LINEAR_BWD, &g, &p, &drop);
    if (rc) return rc;
    if (!buf || buf_len == 0) return fail(CAC_ERR_INVALID_ARG, "buf is NULL or empty");
    int n = snprintf(buf, buf_len, "X %s, W %s", p.pack_x ? "packed" : "as it lies", p.pack_w ? "packed" : "as it lies");
    auto more = [&](const char *fmt, const char *tile, int slices) {
        if (n > 0 && (size_t)n < buf_len) n += snprintf(buf + n, buf_len - n, fmt, tile, slices);
    };
    if ((op == CAC_LINEAR_FWD || p.again) && p.few) more("; pre-activation: %s%.0d", "few rows", 0);
    else if (op == CAC_LINEAR_FWD || p.again) more("; pre-activation: tile %s in %d slices", kTiles[p.y.shape], p.y.slices);
    if (op == CAC_LINEAR_BWD) {
        more("; dX: tile %s in %d slices", kTiles[p.dx.shape], p.dx.slices);
        more("; dW: tile %s in %d slices", kTiles[p.dw.shape], p.dw.slices);
    }
    return CAC_OK;
}

int cac_linear_fwd(const cac_linear_desc *d, const void *X, const void *W, const void *b, const void *R, const uint64_t *rng, void *Y, void *ws,
                   size_t ws_bytes, void *stream)
{
    LinearGeom g;
    LinearPlan p;
    Drop drop;
    int rc = make_linear(d, false, &g, &p, &drop);
    if (rc) return rc;
    if ((rc = check_ptr(X, "X")) || (rc = check_ptr(W, "W")) || (rc = check_ptr(Y, "Y")) || (rc = check_optional(R, "R")) || (rc = check_rng(drop, rng)))
        return rc;
    if (g.bias && (rc = check_ptr(b, "b"))) return rc;
    if ((rc = check_ws(p.bytes, ws, ws_bytes))) return rc;
    drop.rng = rng;
    const size_t e = bytes_of(g.dtype);
    const bool in_place = Y == R && g.ld_r == g.N;
    const Buffer buffers[] = {{Y, g.T * g.N * e, "Y"}, {X, rows_bytes(g.T, g.D, g.ld_x, e), "X"}, {W, rows_bytes(g.N, g.D, g.ld_w, e), "W"},
                              {g.bias ? b : nullptr, g.N * e, "b"}, {in_place ? nullptr : R, rows_bytes(g.T, g.N, g.ld_r, e), "R"},
                              {drop.limit ? rng : nullptr, 16, "rng"}, {ws, p.bytes, "the workspace"}};
    if ((rc = check_apart(buffers, 1, 7))) return rc;
    return launched(launch_linear_fwd(g, p, drop, X, W, g.bias ? b : nullptr, R, Y, ws, (hipStream_t)stream), "linear");
}

int cac_linear_bwd(const cac_linear_desc *d, const void *X, const void *W, const void *b, const void *dY, const uint64_t *rng, void *dX, void *dW, void *db,
                   void *ws, size_t ws_bytes, void *stream)
{
    LinearGeom g;
    LinearPlan p;
    Drop drop;
    int rc = make_linear(d, true, &g, &p, &drop);
    if (rc) return rc;
    if (!dX && !dW && !db) return fail(CAC_ERR_INVALID_ARG, "dX, dW and db are all NULL: nothing to compute");
    const bool need_x = p.again || dW, need_w = p.again || dX, need_b = p.again && g.bias;
    if ((need_x && (rc = check_ptr(X, "X"))) || (need_w && (rc = check_ptr(W, "W"))) || (need_b && (rc = check_ptr(b, "b"))) ||
        (rc = check_ptr(dY, "dY")) || (rc = check_rng(drop, rng)) || (rc = check_optional(dX, "dX")) || (rc = check_optional(dW, "dW")) ||
        (rc = check_optional(db, "db")))
        return rc;
    if ((rc = check_ws(p.bytes, ws, ws_bytes))) return rc;
    drop.rng = rng;
    const size_t e = bytes_of(g.dtype);
    const Buffer buffers[] = {{dX, g.T * g.D * e, "dX"}, {dW, g.N * g.D * e, "dW"}, {db, g.N * e, "db"},
                              {need_x ? X : nullptr, rows_bytes(g.T, g.D, g.ld_x, e), "X"}, {need_w ? W : nullptr, rows_bytes(g.N, g.D, g.ld_w, e), "W"},
                              {need_b ? b : nullptr, g.N * e, "b"}, {dY, g.T * g.N * e, "dY"}, {drop.limit ? rng : nullptr, 16, "rng"},
                              {ws, p.bytes, "the workspace"}};
    if ((rc = check_apart(buffers, 3, 9))) return rc;
    return launched(launch_linear_bwd(g, p, drop, X, W, need_b ? b : nullptr, dY, dX, dW, db, ws, (hipStream_t)stream), "linear backward");
}

int cac_dropout(const cac_dropout_desc *d, const void *X, const void *R, const uint64_t *rng, void *Y, void *stream)
{
    if (!d) return fail(CAC_ERR_INVALID_ARG, "descriptor is NULL");
    Drop drop;
    int rc = check_size(d, d->size, sizeof *d);
    if (rc) return rc;
    if (d->rows <= 0 || d->cols <= 0) return fail(CAC_ERR_INVALID_ARG, "rows and cols must be positive");
    if ((rc = check_dtype(d->dtype))) return rc;
    if ((d->ld_x && d->ld_x < d->cols) || (d->ld_r && d->ld_r < d->cols))
        return fail(CAC_ERR_INVALID_ARG, "ld_x and ld_r are 0 (dense rows) or at least cols");
    if ((rc = make_drop(d->drop_p, d->site, d->alpha, rng, &drop))) return rc;
    DropGeom g;
    g.rows = d->rows;
    g.cols = d->cols;
    g.ld_x = d->ld_x ? d->ld_x : d->cols;
    g.ld_r = d->ld_r ? d->ld_r : d->cols;
    g.dtype = d->dtype;
    g.alpha = d->alpha;
    // a group's number has 40 bits, and a column's 31
    if (g.cols > 1L << 30 || g.rows * ((g.cols + 7) / 8) >= 1L << 40)
        return fail(CAC_ERR_UNSUPPORTED, "cols above 2^30, or 2^40 groups of eight elements or more");
    if ((rc = check_ptr(X, "X")) || (rc = check_optional(R, "R")) || (rc = check_ptr(Y, "Y")) || (rc = check_rng(drop, rng))) return rc;
    const size_t e = bytes_of(g.dtype);
    const bool over_x = Y == X && g.ld_x == g.cols, over_r = Y == R && g.ld_r == g.cols;
    const Buffer buffers[] = {{Y, g.rows * g.cols * e, "Y"}, {over_x ? nullptr : X, rows_bytes(g.rows, g.cols, g.ld_x, e), "X"},
                              {over_r ? nullptr : R, rows_bytes(g.rows, g.cols, g.ld_r, e), "R"}, {drop.limit ? rng : nullptr, 16, "rng"}};
    if ((rc = check_apart(buffers, 1, 4))) return rc;
    return launched(launch_dropout(g, drop, X, R, Y, (hipStream_t)stream), "dropout");
}

int cac_block_norm_workspace_size(const cac_block_norm_desc *d, int op, size_t *bytes)
{
    NormGeom g;
    NormPlan p;
    Drop drop;
    if (op != CAC_BLOCK_NORM_FWD && op != CAC_BLOCK_NORM_BWD) return fail(CAC_ERR_INVALID_ARG, "unknown op %d", op);
    int rc = make_norm(d, op == CAC_BLOCK_NORM_BWD, &g, &p, &drop);
    if (rc) return rc;
    if (!bytes) return fail(CAC_ERR_INVALID_ARG, "bytes is NULL");
    *bytes = p.bytes;
    return CAC_OK;
}

int cac_block_norm_describe_plan(const cac_block_norm_desc *d, int op, char *buf, size_t buf_len)
{
    NormGeom g;
    NormPlan p;
    Drop drop;
    if (op != CAC_BLOCK_NORM_FWD && op != CAC_BLOCK_NORM_BWD) return fail(CAC_ERR_INVALID_ARG, "unknown op %d", op);
    int rc = make_norm(d, op == CAC_BLOCK_NORM_BWD, &g, &p, &drop);
    if (rc) return rc;
    if (!buf || buf_len == 0) return fail(CAC_ERR_INVALID_ARG, "buf is NULL or empty");
    snprintf(buf, buf_len, "%ld workgroups, %d rows at once of %d lanes, %d groups of eight to a lane%s", p.split.blocks, p.slots, p.lanes * p.waves, p.chunks,
             p.two ? ", sums by themselves" : "");
    return CAC_OK;
}

int cac_block_norm_fwd(const cac_block_norm_desc *d, const void *F, const void *R, const float *gate, const float *w_post, const float *b_post,
                       const float *w_pre, const float *b_pre, const uint64_t *rng, void *S, void *H, void *stream)
{
    NormGeom g;
    NormPlan p;
    Drop drop;
    int rc = make_norm(d, false, &g, &p, &drop);
    if (rc) return rc;
    const bool post = g.post != CAC_NORM_NONE, pre = g.pre != CAC_NORM_NONE;
    if (!S && !H) return fail(CAC_ERR_INVALID_ARG, "S and H are both NULL: nothing to compute");
    if ((rc = check_ptr(F, "F")) || (rc = check_optional(R, "R")) || (rc = check_optional(S, "S")) || (rc = check_rng(drop, rng)) ||
        (rc = g.gate_rows ? check_ptr(gate, "gate") : check_absent(gate, "gate", "gate_rows is 0")) ||
        (rc = post ? check_optional(w_post, "w_post") : check_absent(w_post, "w_post", "post is no norm")) ||
        (rc = post ? check_optional(b_post, "b_post") : check_absent(b_post, "b_post", "post is no norm")) ||
        (rc = pre ? check_optional(w_pre, "w_pre") : check_absent(w_pre, "w_pre", "pre is no norm")) ||
        (rc = pre ? check_optional(b_pre, "b_pre") : check_absent(b_pre, "b_pre", "pre is no norm")) ||
        (rc = pre ? check_ptr(H, "H") : check_absent(H, "H", "pre is no norm")))
        return rc;
    drop.rng = rng;
    const size_t e = bytes_of(g.dtype), whole = g.T * g.D * e, vec = g.D * 4;
    const bool in_place = S == R && g.ld_r == g.D;
    const Buffer buffers[] = {{S, whole, "S"}, {H, whole, "H"}, {F, rows_bytes(g.T, g.D, g.ld_f, e), "F"},
                              {in_place ? nullptr : R, rows_bytes(g.T, g.D, g.ld_r, e), "R"}, {gate, p.groups * vec, "gate"}, {w_post, vec, "w_post"},
                              {b_post, vec, "b_post"}, {w_pre, vec, "w_pre"}, {b_pre, vec, "b_pre"}, {drop.limit ? rng : nullptr, 16, "rng"}};
    if ((rc = check_apart(buffers, 2, 10))) return rc;
    return launched(launch_norm_fwd(g, p, drop, F, R, NormParams{gate, w_post, b_post, w_pre, b_pre}, S, H, (hipStream_t)stream), "block norm");
}

int cac_block_norm_bwd(const cac_block_norm_desc *d, const void *F, const void *S, const float *gate, const float *w_post, const float *b_post,
                       const float *w_pre, const void *dH, const void *dS, const uint64_t *rng, void *dR, void *dF, float *dgate, float *dw_post,
                       float *db_post, float *dw_pre, float *db_pre, void *ws, size_t ws_bytes, void *stream)
{
    NormGeom g;
    NormPlan p;
    Drop drop;
    int rc = make_norm(d, true, &g, &p, &drop);
    if (rc) return rc;
    const bool post = g.post != CAC_NORM_NONE, pre = g.pre != CAC_NORM_NONE, need_f = post || g.gate_rows;
    if (!dR && !dF && !dgate && !dw_post && !db_post && !dw_pre && !db_pre)
        return fail(CAC_ERR_INVALID_ARG, "every gradient is NULL: nothing to compute");
    if (!pre && !dS) return fail(CAC_ERR_INVALID_ARG, "dS is NULL and pre is no norm: there is no gradient to start from");
    if ((need_f && (rc = check_ptr(F, "F"))) || (pre && (rc = check_ptr(S, "S"))) ||
        (rc = pre ? check_ptr(dH, "dH") : check_absent(dH, "dH", "pre is no norm")) || (rc = check_optional(dS, "dS")) || (rc = check_rng(drop, rng)) ||
        (rc = g.gate_rows ? check_ptr(gate, "gate") : check_absent(gate, "gate", "gate_rows is 0")) ||
        (rc = g.gate_rows ? check_optional(dgate, "dgate") : check_absent(dgate, "dgate", "gate_rows is 0")) ||
        (rc = post ? check_optional(w_post, "w_post") : check_absent(w_post, "w_post", "post is no norm")) ||
        (rc = post ? check_optional(b_post, "b_post") : check_absent(b_post, "b_post", "post is no norm")) ||
        (rc = pre ? check_optional(w_pre, "w_pre") : check_absent(w_pre, "w_pre", "pre is no norm")) ||
        (rc = post ? check_optional(dw_post, "dw_post") : check_absent(dw_post, "dw_post", "post is no norm")) ||
        (rc = post ? check_optional(db_post, "db_post") : check_absent(db_post, "db_post", "post is no norm")) ||
        (rc = pre ? check_optional(dw_pre, "dw_pre") : check_absent(dw_pre, "dw_pre", "pre is no norm")) ||
        (rc = pre ? check_optional(db_pre, "db_pre") : check_absent(db_pre, "db_pre", "pre is no norm")) || (rc = check_optional(dR, "dR")) ||
        (rc = check_optional(dF, "dF")))
        return rc;
    if ((rc = check_ws(p.bytes, ws, ws_bytes))) return rc;
    drop.rng = rng;
    const size_t e = bytes_of(g.dtype), whole = g.T * g.D * e, vec = g.D * 4;
    const bool once = !p.two, over_s = once && dR && dR == dS, over_f = once && dF && dF == F && g.ld_f == g.D; // (else they are read again)
    const Buffer buffers[] = {{dR, whole, "dR"}, {dF, whole, "dF"}, {dgate, p.groups * vec, "dgate"}, {dw_post, vec, "dw_post"},
                              {db_post, vec, "db_post"}, {dw_pre, vec, "dw_pre"}, {db_pre, vec, "db_pre"},
                              {need_f && !over_f ? F : nullptr, rows_bytes(g.T, g.D, g.ld_f, e), "F"}, {pre ? S : nullptr, whole, "S"}, {dH, whole, "dH"},
                              {over_s ? nullptr : dS, whole, "dS"}, {gate, p.groups * vec, "gate"}, {w_post, vec, "w_post"}, {b_post, vec, "b_post"},
                              {w_pre, vec, "w_pre"}, {drop.limit ? rng : nullptr, 16, "rng"}, {ws, p.bytes, "the workspace"}};
    if ((rc = check_apart(buffers, 7, 17))) return rc;
    return launched(launch_norm_bwd(g, p, drop, need_f ? F : nullptr, pre ? S : nullptr, NormParams{gate, w_post, b_post, w_pre, nullptr}, dH, dS, dR, dF,
                                    NormGrads{dgate, dw_post, db_post, dw_pre, db_pre}, ws, (hipStream_t)stream),
                    "block norm backward");
}

} // extern "C"
