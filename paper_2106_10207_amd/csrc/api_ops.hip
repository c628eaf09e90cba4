// C ABI of the model-step operators (declared in include/dedloc.h): argument
// validation, the matrices' regions of the workspace and the launch sequences.
// All arithmetic on their data runs in ortho.hip and embed.hip.
#include <math.h>
#include <string.h>

#include <algorithm>

#include "../../include/dedloc.h"
#include "api_common.h"
#include "ops_internal.h"

using namespace dedloc;

static_assert((int)kF32 == DEDLOC_DTYPE_F32 && (int)kFP16 == DEDLOC_DTYPE_FP16 && (int)kBF16 == DEDLOC_DTYPE_BF16, "");
static_assert(kNsMaxShort == DEDLOC_ORTHO_MAX_SHORT && kNsMaxLong == DEDLOC_ORTHO_MAX_LONG, "");

namespace {

#ifndef NS_TI
#define NS_TI 128
#define NS_TJ 256
#endif
#ifndef NS_FEW
#define NS_FEW 256
#endif
constexpr uint32_t kNsFewTiles = NS_FEW;

uint32_t blocks(uint64_t n, uint32_t per) { return (uint32_t)((n + per - 1) / per); }

int check_sides(uint32_t k, uint32_t rows, uint32_t cols) {
    if (std::min(rows, cols) > kNsMaxShort || std::max(rows, cols) > kNsMaxLong)
        return fail(DEDLOC_ERR_INVALID_ARG, "matrix %u (%u x %u) exceeds %u by %u", k, rows, cols, kNsMaxShort, kNsMaxLong);
    return DEDLOC_OK;
}

int check_ortho(const dedloc_ortho_cfg &c) {
    if (c.steps == 0 || c.steps > DEDLOC_ORTHO_MAX_STEPS)
        return fail(DEDLOC_ERR_INVALID_ARG, "steps must be in [1, %d] (got %u)", DEDLOC_ORTHO_MAX_STEPS, c.steps);
    return DEDLOC_OK;
}

// Matrices are worked on in batches of kNsMats, one after the other on the
// same workspace.  A batch is built by add() until it is full.
struct Batch {
    NsTable t;
    uint64_t regions = 0;
    bool muon;
    explicit Batch(bool muon_) : muon(muon_) { clear(); }
    void clear() {
        memset(&t, 0, sizeof t);
        regions = 0;
    }
    bool full() const { return t.n == (uint32_t)kNsMats; }
    static uint32_t S(const NsMat &m) { return blocks(std::min(m.rows, m.cols), kNsPad) * kNsPad; }
    static uint32_t L(const NsMat &m) { return blocks(std::max(m.rows, m.cols), kNsPad) * kNsPad; }
    uint32_t sums(const NsMat &m) const {
        return muon ? blocks((uint64_t)m.rows * m.cols, kSumChunk) : blocks(m.rows, kNsTile) * blocks(m.cols, kNsTile);
    }
    void add(NsMat m) {
        m.base = regions;
        m.part = t.parts;
        const uint64_t s = S(m), l = L(m);
        regions += round_up((size_t)(3 * s * l + 2 * s * s) * 4, 256);
        t.parts += sums(m);
        t.m[t.n++] = m;
    }
    size_t bytes() const { return (size_t)regions + round_up((size_t)t.parts * sizeof(double), 256); }
    // Workgroups of a launch in which matrix m takes count(m).
    template <typename F>
    uint32_t spread(F count) {
        uint32_t g = 0;
        for (uint32_t k = 0; k < t.n; k++) {
            t.m[k].begin = g;
            g += count(t.m[k]);
        }
        return g;
    }
};

// The steps on a batch.  src: where the matrices come from; out: where the
// results go (a dtype, or kNsMuonF32).
int run_batch(Batch &b, int src, int out, const dedloc_ortho_cfg &c, NsArgs a, void *ws, hipStream_t s) {
    if (b.t.n == 0) return DEDLOC_OK;
    a.ws = (char *)ws;
    a.part = (double *)((char *)ws + b.regions);
    a.a = c.a;
    a.b = c.b;
    a.c = c.c;
    a.eps = c.eps;
    uint32_t g = b.spread([&](const NsMat &m) { return b.sums(m); });
    hipError_t e = timed(b.muon ? K_MUON_SUM : K_NS_SUM, s, [&] { return launch_ns_sum(src, b.t, a, g, s); });
    if (e != hipSuccess) return hip_fail(e, "norm launch");
    g = b.spread([&](const NsMat &m) { return blocks(m.rows, kNsPad) * blocks(m.cols, kNsPad); });
    e = timed(K_NS_PREPARE, s, [&] { return launch_ns_prepare(src, b.t, a, g, s); });
    if (e != hipSuccess) return hip_fail(e, "prepare launch");
    // workgroups of a phase in tiles of 128 x 256, or of 64 x 64
    auto tiles = [&](int phase, bool wide) {
        return b.spread([&](const NsMat &m) {
            const uint32_t down = blocks(Batch::S(m), wide ? NS_TI : 64);
            if (phase == kNsApply) return down * blocks(Batch::L(m), wide ? NS_TJ : 64);
            const uint32_t R = wide ? NS_TJ / NS_TI : 1, u = down / R;  // R tile rows have the same number of tiles
            return R * u * (u + 1) / 2 + (down % R) * (u + 1);
        });
    };
    static const int kinds[] = {K_NS_GRAM, K_NS_SQUARE, K_NS_APPLY};
    for (uint32_t k = 0; k < c.steps; k++) {
        a.turn = k % 2;
        a.last = k + 1 == c.steps;
        for (int phase = kNsGram; phase <= kNsApply; phase++) {
            bool wide = true;
            g = tiles(phase, wide);
            if (g < kNsFewTiles) g = tiles(phase, wide = false);
            e = timed(kinds[phase], s, [&] { return launch_ns_product(phase, out, wide, b.t, a, g, s); });
            if (e != hipSuccess) return hip_fail(e, "product launch");
        }
    }
    return DEDLOC_OK;
}

int check_ws(const void *ws, size_t have, size_t need) {
    if (!ws || have < need)
        return fail(DEDLOC_ERR_WORKSPACE, "workspace of %zu bytes needed (got %zu)", need, ws ? have : (size_t)0);
    if (!aligned(ws, 256)) return fail(DEDLOC_ERR_ALIGN, "workspace must be 256-byte aligned");
    return DEDLOC_OK;
}

// Workspace of matrices given by their sides: the largest batch's.
template <typename F>
size_t batches_bytes(bool muon, uint32_t n, F sides) {
    Batch b(muon);
    size_t most = 256;
    for (uint32_t k = 0; k < n; k++) {
        NsMat m = {};
        sides(k, m.rows, m.cols);
        if (m.rows == 0 || m.cols == 0) continue;
        if (check_sides(k, m.rows, m.cols)) return 0;
        if (b.full()) b.clear();
        b.add(m);
        most = std::max(most, b.bytes());
    }
    return most;
}

// ------------------------------------------------ embedding and its gradient

struct EmbedWs {
    size_t pairs, counts, total;
    uint32_t chunk;
};
EmbedWs embed_ws(uint64_t n, uint32_t width) {
    EmbedWs w;
    w.pairs = round_up((size_t)n * sizeof(uint2), 256);
    const uint32_t tiles = std::max(1u, blocks(n, kSortTile));
    w.chunk = (tiles + kSortChunks - 1) / kSortChunks * kSortTile;
    w.counts = (size_t)blocks(n, w.chunk) * 256 * sizeof(uint32_t);
    w.total = 2 * w.pairs + w.counts + round_up((size_t)blocks(n, kRunChunk) * 2 * width * sizeof(float), 256);
    w.total = std::max(w.total, (size_t)256);
    return w;
}

int check_embed_sizes(uint64_t n, uint64_t vocab, uint32_t width) {
    if (n > kEmbedMaxTokens) return fail(DEDLOC_ERR_INVALID_ARG, "n must be at most 2^30 (got %llu)", (unsigned long long)n);
    if (vocab > kEmbedMaxVocab) return fail(DEDLOC_ERR_INVALID_ARG, "vocab must be at most 2^30 (got %llu)", (unsigned long long)vocab);
    if (width > kEmbedMaxWidth) return fail(DEDLOC_ERR_INVALID_ARG, "width must be at most 2^20 (got %u)", width);
    return DEDLOC_OK;
}

int check_rows(const void *p, int32_t dtype, uint64_t rows, uint32_t width, uint64_t ld, const char *name) {
    if (dtype != DEDLOC_DTYPE_F32 && dtype != DEDLOC_DTYPE_FP16 && dtype != DEDLOC_DTYPE_BF16)
        return fail(DEDLOC_ERR_INVALID_ARG, "%s: unknown dtype %d", name, dtype);
    if (rows == 0 || width == 0) return DEDLOC_OK;
    if (!p) return fail(DEDLOC_ERR_INVALID_ARG, "%s must not be NULL", name);
    if (!aligned(p, dtype == DEDLOC_DTYPE_F32 ? 4 : 2)) return fail(DEDLOC_ERR_ALIGN, "%s must be aligned to its elements", name);
    if (ld < width) return fail(DEDLOC_ERR_INVALID_ARG, "%s: a row stride is less than the width", name);
    return DEDLOC_OK;
}

int check_embed(const void *table, int32_t table_dtype, uint64_t vocab, uint32_t width, uint64_t ld_table, const void *ids,
                int32_t id_bytes, uint64_t n, const void *rows, int32_t rows_dtype, uint64_t ld_rows,
                const char *table_name, const char *rows_name) {
    int rc = check_embed_sizes(n, vocab, width);
    if (rc) return rc;
    if (id_bytes != 4 && id_bytes != 8) return fail(DEDLOC_ERR_INVALID_ARG, "id_bytes must be 4 or 8 (got %d)", id_bytes);
    rc = check_rows(table, table_dtype, n ? vocab : 0, width, ld_table, table_name);
    if (rc) return rc;
    rc = check_rows(rows, rows_dtype, n, width, ld_rows, rows_name);
    if (rc) return rc;
    if (n && width && !ids) return fail(DEDLOC_ERR_INVALID_ARG, "ids must not be NULL");
    if (!aligned(ids, (size_t)id_bytes)) return fail(DEDLOC_ERR_ALIGN, "ids must be aligned to their elements");
    return DEDLOC_OK;
}

}  // namespace

extern "C" {

size_t dedloc_orthogonalize_workspace_bytes(const dedloc_matrix *mats, uint32_t n) {
    if (!mats || n == 0) {
        fail(DEDLOC_ERR_INVALID_ARG, "mats must list n >= 1 matrices");
        return 0;
    }
    return batches_bytes(false, n, [&](uint32_t k, uint32_t &r, uint32_t &c) {
        r = mats[k].rows;
        c = mats[k].cols;
    });
}

int dedloc_orthogonalize(const dedloc_matrix *mats, uint32_t n, int32_t dtype, const dedloc_ortho_cfg *cfg,
                         void *ws, size_t ws_bytes, void *stream) {
    if (!mats || n == 0) return fail(DEDLOC_ERR_INVALID_ARG, "mats must list n >= 1 matrices");
    if (!cfg) return fail(DEDLOC_ERR_INVALID_ARG, "cfg must not be NULL");
    if (dtype != DEDLOC_DTYPE_F32 && dtype != DEDLOC_DTYPE_FP16 && dtype != DEDLOC_DTYPE_BF16)
        return fail(DEDLOC_ERR_INVALID_ARG, "unknown dtype %d", dtype);
    int rc = check_ortho(*cfg);
    if (rc) return rc;
    const size_t size = dtype == DEDLOC_DTYPE_F32 ? 4 : 2;
    for (uint32_t k = 0; k < n; k++) {
        const dedloc_matrix &m = mats[k];
        if (m.rows == 0 || m.cols == 0) continue;
        rc = check_sides(k, m.rows, m.cols);
        if (rc) return rc;
        if (!m.in || !m.out) return fail(DEDLOC_ERR_INVALID_ARG, "matrix %u: in and out must not be NULL", k);
        if (m.ld_in < m.cols || m.ld_out < m.cols)
            return fail(DEDLOC_ERR_INVALID_ARG, "matrix %u: a row stride is less than its %u columns", k, m.cols);
        if (!aligned(m.in, size) || !aligned(m.out, size))
            return fail(DEDLOC_ERR_ALIGN, "matrix %u: pointers must be aligned to their elements", k);
    }
    const size_t need = dedloc_orthogonalize_workspace_bytes(mats, n);
    if (need == 0) return DEDLOC_ERR_INVALID_ARG;
    rc = check_ws(ws, ws_bytes, need);
    if (rc) return rc;
    Batch b(false);
    NsArgs a = {};
    for (uint32_t k = 0; k < n; k++) {
        const dedloc_matrix &q = mats[k];
        if (q.rows == 0 || q.cols == 0) continue;
        if (b.full()) {
            rc = run_batch(b, dtype, dtype, *cfg, a, ws, (hipStream_t)stream);
            if (rc) return rc;
            b.clear();
        }
        NsMat m = {};
        m.in = q.in;
        m.out = q.out;
        m.ld_in = q.ld_in;
        m.ld_out = q.ld_out;
        m.rows = q.rows;
        m.cols = q.cols;
        b.add(m);
    }
    return run_batch(b, dtype, dtype, *cfg, a, ws, (hipStream_t)stream);
}

size_t dedloc_muon_workspace_bytes(const uint32_t *rows, const uint32_t *cols, uint32_t n_tensors) {
    if (!rows || !cols || n_tensors == 0) {
        fail(DEDLOC_ERR_INVALID_ARG, "rows and cols must list n_tensors >= 1 tensors");
        return 0;
    }
    return batches_bytes(true, n_tensors, [&](uint32_t k, uint32_t &r, uint32_t &c) {
        r = rows[k];
        c = cols[k];
    });
}

int dedloc_muon_step(float *x, float *m, const void *grad, const float *grad_scales, int32_t grad_codec,
                     uint32_t block, uint64_t P, const uint64_t *offsets, const uint32_t *rows, const uint32_t *cols,
                     const uint8_t *flags, uint32_t n_tensors, const dedloc_muon_cfg *cfg, void *ws, size_t ws_bytes,
                     void *stream) {
    if (!cfg) return fail(DEDLOC_ERR_INVALID_ARG, "cfg must not be NULL");
    int rc = check_ortho(cfg->ortho);
    if (rc) return rc;
    if (grad_codec != DEDLOC_CODEC_F32 && grad_codec != DEDLOC_CODEC_FP16 && grad_codec != DEDLOC_CODEC_I8)
        return fail(DEDLOC_ERR_INVALID_ARG, "unknown codec %d", grad_codec);
    if (grad_codec == DEDLOC_CODEC_I8 && block != DEDLOC_I8_BLOCK)
        return fail(DEDLOC_ERR_INVALID_ARG, "int8 block must be %d (got %u)", DEDLOC_I8_BLOCK, block);
    if (!offsets || !rows || !cols || !flags || n_tensors == 0)
        return fail(DEDLOC_ERR_INVALID_ARG, "offsets, rows, cols and flags must list n_tensors >= 1 tensors");
    if (offsets[0] != 0 || offsets[n_tensors] != P)
        return fail(DEDLOC_ERR_INVALID_ARG, "tensor offsets must start at 0 and end at P");
    for (uint32_t k = 0; k < n_tensors; k++) {
        if (offsets[k + 1] < offsets[k]) return fail(DEDLOC_ERR_INVALID_ARG, "tensor offsets decrease at %u", k);
        if (offsets[k] % 8) return fail(DEDLOC_ERR_ALIGN, "tensor offset %u is not a multiple of 8", k);
        if (rows[k] == 0 || cols[k] == 0) continue;
        rc = check_sides(k, rows[k], cols[k]);
        if (rc) return rc;
        const uint64_t len = offsets[k + 1] - offsets[k], n = (uint64_t)rows[k] * cols[k];
        if (len < n || len - n > 7)
            return fail(DEDLOC_ERR_INVALID_ARG, "tensor %u holds %llu elements, %u x %u need %llu (and at most 7 more)", k,
                        (unsigned long long)len, rows[k], cols[k], (unsigned long long)n);
    }
    if (P > 0 && (!x || !m || !grad)) return fail(DEDLOC_ERR_INVALID_ARG, "x, m and grad must not be NULL");
    if (!aligned(x, 16) || !aligned(m, 16) || !aligned(grad, 16))
        return fail(DEDLOC_ERR_ALIGN, "x, m and grad must be 16-byte aligned");
    if (P > 0 && grad_codec == DEDLOC_CODEC_I8 && (!grad_scales || !aligned(grad_scales, 4)))
        return fail(DEDLOC_ERR_INVALID_ARG, "int8 gradient needs aligned grad_scales");
    const size_t need = dedloc_muon_workspace_bytes(rows, cols, n_tensors);
    if (need == 0) return DEDLOC_ERR_INVALID_ARG;
    rc = check_ws(ws, ws_bytes, need);
    if (rc) return rc;
    const int src = grad_codec == DEDLOC_CODEC_F32 ? kNsMuonF32 : grad_codec == DEDLOC_CODEC_FP16 ? kNsMuonFP16 : kNsMuonI8;
    Batch b(true);
    NsArgs a = {};
    a.x = x;
    a.mom = m;
    a.grad = grad;
    a.scales = grad_scales;
    a.mu = cfg->momentum;
    a.keep = (float)(1.0 - (double)cfg->lr * (double)cfg->weight_decay);
    a.nesterov = cfg->nesterov;
    for (uint32_t k = 0; k < n_tensors; k++) {
        if (rows[k] == 0 || cols[k] == 0) continue;
        if (b.full()) {
            rc = run_batch(b, src, kNsMuonF32, cfg->ortho, a, ws, (hipStream_t)stream);
            if (rc) return rc;
            b.clear();
        }
        NsMat q = {};
        q.ld_in = offsets[k];
        q.rows = rows[k];
        q.cols = cols[k];
        q.flags = flags[k];
        const double ratio = flags[k] & DEDLOC_TENSOR_ADAPT ? (double)cfg->rms * sqrt((double)std::max(rows[k], cols[k])) : 1.0;
        q.unit = (float)((double)cfg->lr * ratio);
        b.add(q);
    }
    return run_batch(b, src, kNsMuonF32, cfg->ortho, a, ws, (hipStream_t)stream);
}

int dedloc_embed(const void *table, int32_t table_dtype, uint64_t vocab, uint32_t width, uint64_t ld_table,
                 const void *ids, int32_t id_bytes, uint64_t n, float scale, void *out, int32_t out_dtype,
                 uint64_t ld_out, void *stream) {
    int rc = check_embed(table, table_dtype, vocab, width, ld_table, ids, id_bytes, n, out, out_dtype, ld_out, "table", "out");
    if (rc) return rc;
    if (n == 0 || width == 0) return DEDLOC_OK;
    const EmbedArgs a = {table, ld_table, ids, out, ld_out, (uint32_t)vocab, width, (uint32_t)n, id_bytes == 8, scale};
    hipStream_t s = (hipStream_t)stream;
    const hipError_t e = timed(K_EMBED, s, [&] { return launch_embed(table_dtype, out_dtype, a, s); });
    return e == hipSuccess ? DEDLOC_OK : hip_fail(e, "embed launch");
}

size_t dedloc_embed_workspace_bytes(uint64_t n, uint64_t vocab, uint32_t width) {
    if (check_embed_sizes(n, vocab, width)) return 0;
    return embed_ws(n, width).total;
}

int dedloc_embed_grad(float *grad, uint64_t vocab, uint32_t width, uint64_t ld_grad, const void *ids, int32_t id_bytes,
                      uint64_t n, const void *dy, int32_t dy_dtype, uint64_t ld_dy, float scale, float batch_samples,
                      void *ws, size_t ws_bytes, void *stream) {
    int rc = check_embed(grad, DEDLOC_DTYPE_F32, vocab, width, ld_grad, ids, id_bytes, n, dy, dy_dtype, ld_dy, "grad", "dy");
    if (rc) return rc;
    if (n == 0 || width == 0 || vocab == 0) return DEDLOC_OK;
    const EmbedWs w = embed_ws(n, width);
    rc = check_ws(ws, ws_bytes, w.total);
    if (rc) return rc;
    char *b = (char *)ws;
    const EmbedGradArgs a = {grad, ld_grad, ids, dy, ld_dy, (uint32_t)vocab, width, (uint32_t)n, id_bytes == 8,
                             scale * batch_samples, w.chunk, {(uint2 *)b, (uint2 *)(b + w.pairs)}, (uint32_t *)(b + 2 * w.pairs),
                             (float *)(b + 2 * w.pairs + w.counts)};
    hipStream_t s = (hipStream_t)stream;
    int from = -1;
    // digits of the tokens and of `vocab`, which stands for a masked position
    for (uint32_t shift = 0; shift == 0 || vocab >> shift; shift += 8) {
        hipError_t e = timed(K_EMBED_COUNT, s, [&] { return launch_embed_count(a, from, shift, s); });
        if (e != hipSuccess) return hip_fail(e, "embed count launch");
        e = timed(K_EMBED_SCATTER, s, [&] { return launch_embed_scatter(a, from, shift, s); });
        if (e != hipSuccess) return hip_fail(e, "embed scatter launch");
        from = from < 0 ? 0 : 1 - from;
    }
    hipError_t e = timed(K_EMBED_SUM, s, [&] { return launch_embed_sum(dy_dtype, a, from, s); });
    if (e != hipSuccess) return hip_fail(e, "embed sum launch");
    e = timed(K_EMBED_JOIN, s, [&] { return launch_embed_join(a, from, s); });
    return e == hipSuccess ? DEDLOC_OK : hip_fail(e, "embed join launch");
}

}  // extern "C"
