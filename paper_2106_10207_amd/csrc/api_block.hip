// C ABI of dropout, the norms and the ends of a block (declared in
// include/dedloc.h): argument validation, the workspace and the launches.  All
// arithmetic on their data runs in block.hip.
#include <math.h>

#include <algorithm>

#include "../../include/dedloc.h"
#include "api_common.h"
#include "block_internal.h"

using namespace dedloc;

static_assert((int)kNormNone == DEDLOC_NORM_NONE && (int)kNormLayer == DEDLOC_NORM_LAYER && (int)kNormRms == DEDLOC_NORM_RMS, "");
static_assert(kNormMaxWidth == DEDLOC_NORM_MAX_WIDTH, "");

namespace {

int check_dtype(int32_t dtype, const char *name) {
    if (dtype != DEDLOC_DTYPE_F32 && dtype != DEDLOC_DTYPE_FP16 && dtype != DEDLOC_DTYPE_BF16)
        return fail(DEDLOC_ERR_INVALID_ARG, "%s: unknown dtype %d", name, dtype);
    return DEDLOC_OK;
}

int check_sizes(uint64_t rows, uint32_t width, uint32_t most) {
    if (rows > kBlockMaxRows) return fail(DEDLOC_ERR_INVALID_ARG, "rows must be at most 2^30 (got %llu)", (unsigned long long)rows);
    if (width > most) return fail(DEDLOC_ERR_INVALID_ARG, "width must be at most %u (got %u)", most, width);
    return DEDLOC_OK;
}

size_t size_of(int32_t dtype) { return dtype == DEDLOC_DTYPE_F32 ? 4 : 2; }

// rows of `width` elements at p
int check_matrix(const void *p, int32_t dtype, uint32_t width, uint64_t ld, bool needed, const char *name) {
    if (!p) return needed ? fail(DEDLOC_ERR_INVALID_ARG, "%s must not be NULL", name) : DEDLOC_OK;
    if (!aligned(p, size_of(dtype))) return fail(DEDLOC_ERR_ALIGN, "%s must be aligned to its elements", name);
    if (ld < width) return fail(DEDLOC_ERR_INVALID_ARG, "%s: a row stride is less than the width", name);
    return DEDLOC_OK;
}

int check_types(int32_t stream_dtype, int32_t branch_dtype, const char *stream_name, const char *branch_name) {
    int rc = check_dtype(stream_dtype, stream_name);
    if (!rc) rc = check_dtype(branch_dtype, branch_name);
    if (!rc && stream_dtype != DEDLOC_DTYPE_F32 && stream_dtype != branch_dtype)
        rc = fail(DEDLOC_ERR_INVALID_ARG, "%s of 16 bits goes with %s of the same type", stream_name, branch_name);
    return rc;
}

int check_vector(const float *p, const char *name) {
    return aligned(p, 4) ? DEDLOC_OK : fail(DEDLOC_ERR_ALIGN, "%s must be 4-byte aligned", name);
}

int check_norm(const dedloc_norm_cfg &n, const char *name) {
    if (n.kind == DEDLOC_NORM_NONE) return DEDLOC_OK;
    if (n.kind != DEDLOC_NORM_LAYER && n.kind != DEDLOC_NORM_RMS)
        return fail(DEDLOC_ERR_INVALID_ARG, "%s: unknown kind of norm %d", name, n.kind);
    if (!(n.eps >= 1e-30f) || !(n.eps <= 1e30f)) return fail(DEDLOC_ERR_INVALID_ARG, "%s: eps must be in [1e-30, 1e30]", name);
    int rc = check_vector(n.gain, "gain");
    return rc ? rc : check_vector(n.bias, "bias");
}

// A norm that is left out has no vectors, whatever its struct points to: the kernels and the join ask for the vectors alone.
NormArgs norm_args(const dedloc_norm_cfg &n) {
    if (n.kind == DEDLOC_NORM_NONE) return {};
    return {n.kind, n.eps, n.gain, n.bias};
}

int check_dropout(const dedloc_dropout_cfg &d) {
    if (!(d.p >= 0.0f && d.p <= 1.0f)) return fail(DEDLOC_ERR_INVALID_ARG, "p must be in [0, 1] (got %g)", (double)d.p);
    if (!aligned(d.step_at, 8)) return fail(DEDLOC_ERR_ALIGN, "step_at must be 8-byte aligned");
    return DEDLOC_OK;
}

DropArgs drop_args(const dedloc_dropout_cfg &d) {
    const double t = rint((double)d.p * 65536.0);
    const uint32_t threshold = d.p == 1.0f ? 65536 : (uint32_t)std::min(t, 65535.0);
    return {threshold, threshold < 65536 ? (float)(65536.0 / (65536.0 - threshold)) : 0.0f, (uint32_t)d.seed, (uint32_t)(d.seed >> 32),
            d.site, d.step, d.row0, d.step_at};
}

// Workgroups of a gradient and the rows of each of their teams.  Every workgroup leaves a part of each vector's
// gradient that the join reads: no more of them than run at once, kTurns rows a team where there are enough for kFill waves, and
// one where there are few (8192 rows of 1024 fp16: 4 rows a team 24.1 us, 8 22.6; 1001 rows of 333: 24.6 and 32.7).
struct Split {
    uint32_t groups, turns;
};
Split split_rows(uint32_t rows, const RowShape &r, int mode) {
    constexpr uint32_t kTurns = 8, kFill = 2048;
    const uint32_t most = kSimds * resident(kGradWaves, r.vectors, mode, r.threads) * 64 / r.threads, teams = r.teams();
    const uint32_t fill = std::min((rows + teams - 1) / teams, kFill * 64 / r.threads);
    const uint32_t groups = std::min(most, std::max(fill, (rows + teams * kTurns - 1) / (teams * kTurns)));
    return {groups, (rows + groups * teams - 1) / (groups * teams)};
}

// Floats of the parts, and of the edges, of the largest of all calls of at most these rows and columns, whatever shape
// (one or two vectors a thread) and mode they have.
struct Room {
    size_t parts, edges;
    size_t bytes() const { return std::max((size_t)256, round_up(parts * sizeof(float), 256) + round_up(edges * sizeof(float), 256)); }
};
Room room(uint32_t rows, uint32_t width, bool edges) {
    Room most = {0, 0};
    const auto count = [&](uint32_t w) {
        for (int k = 0; k < 8; k++) {
            const RowShape r = row_shape(w, k & 4 ? 1024 : 512);
            const uint32_t groups = split_rows(rows, r, k & 3).groups;
            most.parts = std::max(most.parts, (size_t)groups * kBlockSums * w);
            if (edges) most.edges = std::max(most.edges, (size_t)groups * r.teams() * 2 * w);
        }
    };
    // the widest row of each shape that is narrower
    for (uint32_t w = 64; w < width; w += w < 512 ? w : 512) count(w);
    count(width);
    return most;
}

int check_ws(const void *ws, size_t bytes, size_t need) {
    if (!ws || bytes < need) return fail(DEDLOC_ERR_WORKSPACE, "workspace too small: %zu bytes given, %zu needed", ws ? bytes : (size_t)0, need);
    if (!aligned(ws, 256)) return fail(DEDLOC_ERR_ALIGN, "workspace must be 256-byte aligned");
    return DEDLOC_OK;
}

int check_block(const dedloc_residual_cfg &c, uint32_t width, int32_t branch_dtype) {
    int rc = check_norm(c.post, "post");
    if (!rc) rc = check_norm(c.pre, "pre");
    if (!rc) rc = check_dropout(c.drop);
    if (!rc && c.gate_rows && !c.gate) rc = fail(DEDLOC_ERR_INVALID_ARG, "gate_rows without a gate");
    if (!rc && c.gate_rows) rc = check_matrix(c.gate, branch_dtype, width, c.ld_gate, true, "gate");
    if (!rc && !c.gate_rows) rc = check_vector((const float *)c.gate, "gate");
    return rc;
}

int check_stats(const float *stats, bool needed) {
    if (needed && !stats) return fail(DEDLOC_ERR_INVALID_ARG, "stats must not be NULL");
    return aligned(stats, 8) ? DEDLOC_OK : fail(DEDLOC_ERR_ALIGN, "stats must be 8-byte aligned");
}

// A gradient of a vector that is not there.
int check_grad(const float *grad, bool exists, const char *name) {
    if (grad && !exists) return fail(DEDLOC_ERR_INVALID_ARG, "%s: no such parameter in this call", name);
    return check_vector(grad, name);
}

int run_grad(ResidualGradArgs &a, int32_t stream_dtype, int32_t branch_dtype, void *ws, size_t ws_bytes, hipStream_t s) {
    const bool shared = a.gate && !a.gate_rows;
    a.want = (a.dpre_gain ? 1u : 0u) | (a.dpre_bias ? 2u : 0u) | (a.dpost_gain || (shared && a.dgate) ? 4u : 0u) |
             (a.dpost_bias || (shared && a.dgate && a.post.bias) ? 8u : 0u);
    a.f32 = stream_dtype == DEDLOC_DTYPE_F32;
    const Split split = split_rows(a.rows, grad_shape(a.width, grad_mode(a), a.f32), grad_mode(a));
    a.groups = split.groups;
    a.turns = split.turns;
    const bool cut = a.gate_rows && a.dgate;
    if (a.want || cut) {
        const Room need = room(a.rows, a.width, cut);
        const int rc = check_ws(ws, ws_bytes, need.bytes());
        if (rc) return rc;
        a.part = (float *)ws;
        a.edge = (float *)((char *)ws + round_up(need.parts * sizeof(float), 256));
    }
    hipError_t e = timed(K_RESIDUAL_GRAD, s, [&] { return launch_residual_grad(stream_dtype, branch_dtype, a, s); });
    if (e != hipSuccess) return hip_fail(e, "residual gradient launch");
    if (a.want) {
        e = timed(K_RESIDUAL_JOIN, s, [&] { return launch_residual_join(a, s); });
        if (e != hipSuccess) return hip_fail(e, "residual join launch");
    }
    if (cut) {
        e = timed(K_GATE_JOIN, s, [&] { return launch_gate_join(a, s); });
        if (e != hipSuccess) return hip_fail(e, "gate join launch");
    }
    return DEDLOC_OK;
}

}  // namespace

extern "C" {

int dedloc_dropout(const dedloc_dropout_cfg *cfg, uint64_t rows, uint32_t width, int32_t dtype, const void *x, uint64_t ld_x,
                   void *out, uint64_t ld_out, void *stream) {
    if (!cfg) return fail(DEDLOC_ERR_INVALID_ARG, "cfg must not be NULL");
    int rc = check_sizes(rows, width, kDropMaxWidth);
    if (!rc) rc = check_dtype(dtype, "x");
    if (!rc) rc = check_dropout(*cfg);
    if (rc || rows == 0 || width == 0) return rc;
    rc = check_matrix(x, dtype, width, ld_x, true, "x");
    if (!rc) rc = check_matrix(out, dtype, width, ld_out, true, "out");
    if (rc) return rc;
    const DropoutArgs a = {x, out, ld_x, ld_out, (uint32_t)rows, width, drop_args(*cfg), 0, 0, 0};
    hipStream_t s = (hipStream_t)stream;
    const hipError_t e = timed(K_DROPOUT, s, [&] { return launch_dropout(dtype, a, s); });
    return e == hipSuccess ? DEDLOC_OK : hip_fail(e, "dropout launch");
}

int dedloc_norm(const dedloc_norm_cfg *cfg, uint64_t rows, uint32_t width, int32_t x_dtype, int32_t out_dtype, const void *x,
                uint64_t ld_x, void *out, uint64_t ld_out, float *stats, void *stream) {
    if (!cfg || cfg->kind == DEDLOC_NORM_NONE) return fail(DEDLOC_ERR_INVALID_ARG, "cfg must name a norm");
    int rc = check_sizes(rows, width, kNormMaxWidth);
    if (!rc) rc = check_types(x_dtype, out_dtype, "x", "out");
    if (!rc) rc = check_norm(*cfg, "cfg");
    if (rc || rows == 0 || width == 0) return rc;
    rc = check_matrix(x, x_dtype, width, ld_x, true, "x");
    if (!rc) rc = check_matrix(out, out_dtype, width, ld_out, true, "out");
    if (!rc) rc = check_stats(stats, false);
    if (rc) return rc;
    ResidualArgs a = {};
    a.h = x;
    a.ld_h = ld_x;
    a.out = out;
    a.ld_out = ld_out;
    a.stats = (float2 *)stats;
    a.rows = (uint32_t)rows;
    a.width = width;
    a.pre = norm_args(*cfg);
    hipStream_t s = (hipStream_t)stream;
    const hipError_t e = timed(K_RESIDUAL, s, [&] { return launch_residual(x_dtype, out_dtype, a, s); });
    return e == hipSuccess ? DEDLOC_OK : hip_fail(e, "norm launch");
}

int dedloc_residual(const dedloc_residual_cfg *cfg, uint64_t rows, uint32_t width, int32_t stream_dtype, int32_t branch_dtype,
                    const void *h, uint64_t ld_h, const void *f, uint64_t ld_f, void *sum, uint64_t ld_sum, void *out,
                    uint64_t ld_out, float *stats, void *stream) {
    if (!cfg) return fail(DEDLOC_ERR_INVALID_ARG, "cfg must not be NULL");
    int rc = check_sizes(rows, width, kNormMaxWidth);
    if (!rc) rc = check_types(stream_dtype, branch_dtype, "the stream", "the branch");
    if (!rc) rc = check_block(*cfg, width, branch_dtype);
    if (rc || rows == 0 || width == 0) return rc;
    const bool pre = cfg->pre.kind != DEDLOC_NORM_NONE;
    rc = check_matrix(h, stream_dtype, width, ld_h, true, "h");
    if (!rc) rc = check_matrix(f, branch_dtype, width, ld_f, true, "f");
    if (!rc) rc = check_matrix(sum, stream_dtype, width, ld_sum, !pre, "sum");
    if (!rc && !pre && out) rc = fail(DEDLOC_ERR_INVALID_ARG, "out without a pre norm");
    if (!rc) rc = check_matrix(out, branch_dtype, width, ld_out, pre, "out");
    if (!rc) rc = check_stats(stats, false);
    if (rc) return rc;
    const ResidualArgs a = {h, f, sum, out, (float2 *)stats, ld_h, ld_f, ld_sum, ld_out, cfg->gate, cfg->ld_gate, (uint32_t)rows,
                            width, cfg->gate_rows, cfg->alpha, cfg->beta, norm_args(cfg->post), norm_args(cfg->pre), drop_args(cfg->drop)};
    hipStream_t s = (hipStream_t)stream;
    const hipError_t e = timed(K_RESIDUAL, s, [&] { return launch_residual(stream_dtype, branch_dtype, a, s); });
    return e == hipSuccess ? DEDLOC_OK : hip_fail(e, "residual launch");
}

size_t dedloc_residual_workspace_bytes(uint64_t rows, uint32_t width, uint32_t gate_rows) {
    if (check_sizes(rows, width, kNormMaxWidth)) return 0;
    return room((uint32_t)std::max<uint64_t>(rows, 1), std::max(width, 1u), gate_rows != 0).bytes();
}

int dedloc_norm_grad(const dedloc_norm_cfg *cfg, uint64_t rows, uint32_t width, int32_t x_dtype, int32_t out_dtype, const void *dout,
                     uint64_t ld_dout, const void *x, uint64_t ld_x, const float *stats, const void *add, uint64_t ld_add, void *dx,
                     uint64_t ld_dx, float *dgain, float *dbias, float batch_samples, void *ws, size_t ws_bytes, void *stream) {
    if (!cfg || cfg->kind == DEDLOC_NORM_NONE) return fail(DEDLOC_ERR_INVALID_ARG, "cfg must name a norm");
    int rc = check_sizes(rows, width, kNormMaxWidth);
    if (!rc) rc = check_types(x_dtype, out_dtype, "x", "dout");
    if (!rc) rc = check_norm(*cfg, "cfg");
    if (!rc) rc = check_grad(dgain, cfg->gain, "dgain");
    if (!rc) rc = check_grad(dbias, cfg->bias, "dbias");
    if (rc || rows == 0 || width == 0) return rc;
    rc = check_matrix(dout, out_dtype, width, ld_dout, true, "dout");
    if (!rc) rc = check_matrix(x, x_dtype, width, ld_x, true, "x");
    if (!rc) rc = check_matrix(add, x_dtype, width, ld_add, false, "add");
    if (!rc) rc = check_matrix(dx, x_dtype, width, ld_dx, true, "dx");
    if (!rc) rc = check_stats(stats, true);
    if (rc) return rc;
    ResidualGradArgs a = {};
    a.sum = x;
    a.ld_sum = ld_x;
    a.dsum = add;
    a.ld_dsum = ld_add;
    a.dout = dout;
    a.ld_dout = ld_dout;
    a.dh = dx;
    a.ld_dh = ld_dx;
    a.stats = (const float2 *)stats;
    a.rows = (uint32_t)rows;
    a.width = width;
    a.alpha = 1.0f;
    a.pre = norm_args(*cfg);
    a.dpre_gain = dgain;
    a.dpre_bias = dbias;
    a.samples = batch_samples;
    return run_grad(a, x_dtype, out_dtype, ws, ws_bytes, (hipStream_t)stream);
}

int dedloc_residual_grad(const dedloc_residual_cfg *cfg, uint64_t rows, uint32_t width, int32_t stream_dtype, int32_t branch_dtype,
                         const dedloc_residual_grads *g, float batch_samples, void *ws, size_t ws_bytes, void *stream) {
    if (!cfg || !g) return fail(DEDLOC_ERR_INVALID_ARG, "cfg and grads must not be NULL");
    int rc = check_sizes(rows, width, kNormMaxWidth);
    if (!rc) rc = check_types(stream_dtype, branch_dtype, "the stream", "the branch");
    if (!rc) rc = check_block(*cfg, width, branch_dtype);
    const bool pre = cfg->pre.kind != DEDLOC_NORM_NONE, post = cfg->post.kind != DEDLOC_NORM_NONE;
    if (!rc) rc = check_grad(g->dpre_gain, pre && cfg->pre.gain, "dpre_gain");
    if (!rc) rc = check_grad(g->dpre_bias, pre && cfg->pre.bias, "dpre_bias");
    if (!rc) rc = check_grad(g->dpost_gain, post && cfg->post.gain, "dpost_gain");
    if (!rc) rc = check_grad(g->dpost_bias, post && cfg->post.bias, "dpost_bias");
    if (!rc) rc = check_grad(g->dgate, cfg->gate, "dgate");
    if (!rc && cfg->gate_rows && g->dgate && g->ld_dgate < width)
        rc = fail(DEDLOC_ERR_INVALID_ARG, "dgate: a row stride is less than the width");
    if (rc || rows == 0 || width == 0) return rc;
    const bool reads_f = post || g->dgate;
    rc = check_matrix(g->sum, stream_dtype, width, g->ld_sum, pre, "sum");
    if (!rc) rc = check_matrix(g->f, branch_dtype, width, g->ld_f, reads_f, "f");
    if (!rc && !pre && g->dout) rc = fail(DEDLOC_ERR_INVALID_ARG, "dout without a pre norm");
    if (!rc) rc = check_matrix(g->dout, branch_dtype, width, g->ld_dout, pre, "dout");
    if (!rc) rc = check_matrix(g->dsum, stream_dtype, width, g->ld_dsum, !pre, "dsum");
    if (!rc) rc = check_matrix(g->dh, stream_dtype, width, g->ld_dh, true, "dh");
    if (!rc) rc = check_matrix(g->df, branch_dtype, width, g->ld_df, true, "df");
    if (!rc) rc = check_stats(g->stats, pre || post);
    if (rc) return rc;
    ResidualGradArgs a = {};
    a.sum = g->sum;
    a.ld_sum = g->ld_sum;
    a.f = reads_f ? g->f : nullptr;
    a.ld_f = g->ld_f;
    a.dsum = g->dsum;
    a.ld_dsum = g->ld_dsum;
    a.dout = g->dout;
    a.ld_dout = g->ld_dout;
    a.dh = g->dh;
    a.ld_dh = g->ld_dh;
    a.df = g->df;
    a.ld_df = g->ld_df;
    a.stats = (const float2 *)g->stats;
    a.gate = cfg->gate;
    a.ld_gate = cfg->ld_gate;
    a.gate_rows = cfg->gate_rows;
    a.dgate = g->dgate;
    a.ld_dgate = g->ld_dgate;
    a.rows = (uint32_t)rows;
    a.width = width;
    a.alpha = cfg->alpha;
    a.beta = cfg->beta;
    a.post = norm_args(cfg->post);
    a.pre = norm_args(cfg->pre);
    a.drop = drop_args(cfg->drop);
    a.dpre_gain = g->dpre_gain;
    a.dpre_bias = g->dpre_bias;
    a.dpost_gain = g->dpost_gain;
    a.dpost_bias = g->dpost_bias;
    a.samples = batch_samples;
    return run_grad(a, stream_dtype, branch_dtype, ws, ws_bytes, (hipStream_t)stream);
}

}  // extern "C"
