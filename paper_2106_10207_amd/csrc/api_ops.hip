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

uint32_t padded(uint32_t n) { return blocks(n, kNsPad) * kNsPad; }

// Steps of the block that starts `done` steps into `steps`: how many are taken
// on the s x s side before X is touched again.  An error of A grows by a^2 in each, so a
// block from X0 takes at most three (a = 3.4445: 141 times) and a later one, whose A is no longer
// small, two; with a beyond 3.5 fewer.
uint32_t block_steps(const dedloc_ortho_cfg &c, bool blocked, uint32_t done) {
    if (!blocked) return 1;
    const double grow = (double)c.a * c.a;
    uint32_t n = 1;
    for (double g = grow; g <= 150.0 && n < 3; g *= grow) n++;
    return std::min(done == 0 ? n : std::min(n, 2u), c.steps - done);
}

// The products of a call on one matrix, in order: at most two at a launch.
struct Program {
    uint32_t op[3 * DEDLOC_ORTHO_MAX_STEPS + 64][2];
    uint32_t n = 0;
};
uint32_t op_of(int kind, uint32_t left, uint32_t right, uint32_t out) { return kind | left << 4 | right << 8 | out << 12; }

void make_program(const dedloc_ortho_cfg &c, bool blocked, Program &p) {
    constexpr uint32_t none = ~0u, A0 = kNsSmall, M0 = A0 + 1, A1 = A0 + 2, M1 = A0 + 3, C = A0 + 4, Q = A0 + 5;
    p.n = 0;
    auto add = [&](uint32_t first, uint32_t second = none) {
        p.op[p.n][0] = first;
        p.op[p.n++][1] = second;
    };
    uint32_t turn = 1;  // which X^T is read
    for (uint32_t done = 0; done < c.steps;) {
        const uint32_t n = block_steps(c, blocked, done);
        uint32_t q = M0;
        add(op_of(kNsGram, 0, 0, A0));
        add(op_of(kNsSquare, A0, A0, M0));
        if (n > 1) {
            add(op_of(kNsMul, M0, M0, C));
            add(op_of(kNsMul, C, A0, A1));  // M A M
            add(op_of(kNsSquare, A1, A1, M1));
            if (n == 2) {
                add(op_of(kNsMul, M1, M0, Q));
                q = Q;
            } else {
                add(op_of(kNsMul, M1, M1, C), op_of(kNsMul, M1, M0, Q));
                add(op_of(kNsMul, C, A1, A0));
                add(op_of(kNsSquare, A0, A0, M0));
                add(op_of(kNsMul, M0, Q, M1));
                q = M1;
            }
        }
        done += n;
        add(op_of(done == c.steps ? kNsResult : kNsApply, q, turn, 3 - turn));
        turn = 3 - turn;
    }
}

constexpr uint64_t kNsBlocked = 1ull << 26;
constexpr uint32_t kNarrowMost = 512;  // workgroups

// Whether a matrix is worked on in blocks of steps.  Five steps as blocks of three and two
// are 6 s^2 l + 14 s^3 multiply-adds for 15 s^2 l + 5 s^3, in 17 launches for 15: worth it from
// 9 s^2 (l - s) = 6e8 on.
// The s x s side keeps A's own roundings, which a Gram matrix of a long X averages out: an fp32 result is
// worked on in blocks only up to 4 times as long as wide.  Muon's update of a longer one is left in blocks: 256 x 2304, the
// worst of those timed, is 2.5e-6 off for 1.2e-6 at most (plain fp32 products 1.8e-6), against ResNet-50's matrices in 1013 us for 1200.
bool blocked(uint32_t rows, uint32_t cols, bool fp32) {
    const uint64_t s = std::min(rows, cols), l = std::max(rows, cols);
    return s * s * (l - s) >= kNsBlocked && !(fp32 && l > 4 * s);
}

// Matrices are worked on in batches, one after the other on the same workspace:
// as many as two works each of the blocked ones, one of the others, fit a launch.
struct Batch {
    NsTable t;
    NsWork w[kNsWorks];  // per matrix: the fields that do not change
    bool blocked_[kNsWorks];
    uint32_t works;
    uint64_t regions;
    bool muon, fp32;  // fp32: orthogonalize's results
    Batch(bool muon_, bool fp32_) : muon(muon_), fp32(fp32_) { clear(); }
    void clear() {
        memset(&t, 0, sizeof t);
        works = 0;
        regions = 0;
    }
    bool fits(uint32_t rows, uint32_t cols) const { return works + 1 + blocked(rows, cols, fp32) <= (uint32_t)kNsWorks; }
    uint32_t sums(const NsMat &m) const {
        const uint32_t n = muon ? blocks((uint64_t)m.rows * m.cols, kSumChunk) : blocks(m.rows, kNsTile) * blocks(m.cols, kNsTile);
        return std::min(n, kSumMost);
    }
    void add(const void *in, uint64_t ld_in, void *out, uint64_t ld_out, uint32_t rows, uint32_t cols, uint32_t flags, float unit) {
        const uint64_t s = padded(std::min(rows, cols)), l = padded(std::max(rows, cols));
        const bool b = blocked(rows, cols, fp32);
        NsMat &m = t.m[t.n];
        m = {regions, in, ld_in, rows, cols, t.parts, 0};
        t.parts += sums(m);
        w[t.n] = {regions, out, ld_out, rows, cols, 0, 0, (flags & DEDLOC_TENSOR_DECAY) << 16, unit};
        blocked_[t.n++] = b;
        works += 1 + b;
        regions += round_up((size_t)(kNsSmall * s * l + (b ? kNsSmalls : 2) * s * s) * 4, 256);
    }
    size_t part_bytes() const { return round_up((size_t)t.parts * sizeof(double), 256); }
    // room for the sums of cut items: what a launch cuts stays below it
    size_t piece_bytes() const { return round_up(std::max((size_t)regions / 2, (size_t)4 << 20), 256); }
    size_t bytes() const { return (size_t)regions + part_bytes() + piece_bytes(); }
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
static_assert(DEDLOC_TENSOR_DECAY == 1u, "the flag's bit moves into a work's op");

uint32_t tiles_of(const NsWork &w, uint32_t edge) {
    const uint32_t down = blocks(padded(std::min(w.rows, w.cols)), edge);
    return (w.op & 15) >= kNsApply ? down * blocks(padded(std::max(w.rows, w.cols)), edge) : down * (down + 1) / 2;
}
uint32_t panels_of(const NsWork &w) {
    return padded((w.op & 15) == kNsGram ? std::max(w.rows, w.cols) : std::min(w.rows, w.cols)) / 32;
}
uint32_t pieces_of(uint32_t panels, uint32_t most) { return panels > most + most / 2 ? blocks(panels, most) : 1; }

// How a launch's products are cut: the edge of the tiles, and pieces of at most
// `most` panels of the summed index.
struct Cut {
    uint32_t edge, most;
};

// Estimated time of a launch in us, below 0 if the sums of its cut items take
// more than `room` bytes.  W turns of 32 of the summed index, in `items` tiles of which
// `full` are not symmetric (and written twice), the longest of `longest` turns: bound by
// one workgroup alone on its CU, or by 256 CUs that hold two each; the join
// reads its pieces back.  Fitted to 684 launches (the products of 14 calls of 1 to 54
// matrices, sides of 1 to 8192) timed in tiles of 128 and 64, uncut and in pieces of at most 64,
// 32, 16 and 8 panels.  In all of choose_cut's ways, the 294 launches of 21 calls (those, and sides to 100000): the choice
// by this estimate takes 1.01 of the best times' sum, always 128 uncut 2.3, always 64 uncut 1.5.  145 launches of nine calls
// with sides of 60000 to 15 million, which pieces of 256 and 128 are for: 1.06 (without these two 1.18).
double cost_of(const NsWorks &t, Cut c, size_t room) {
    const bool big = c.edge == 128;
    const double alone = big ? 0.54 : 0.17, once = big ? 9.1 : 5.0, busy = big ? 0.56 : 0.18, item = big ? 4.2 : 2.1,
                 twice = big ? 6.2 : 1.9;
    double W = 0, items = 0, full = 0, cut = 0;
    uint32_t longest = 0;
    for (uint32_t k = 0; k < t.n; k++) {
        const uint32_t P = panels_of(t.w[k]), z = pieces_of(P, c.most);
        const double tiles = tiles_of(t.w[k], c.edge);
        W += tiles * P;
        items += tiles * z;
        if ((t.w[k].op & 15) >= kNsApply) full += tiles;
        if (z > 1) cut += tiles * z * c.edge * c.edge * sizeof(float);
        longest = std::max(longest, blocks(P, z));
    }
    if (cut > (double)room) return -1.0;
    const double filled = (W * busy + items * item + full * twice) / 256 + 0.35 * busy * longest + 5.0;
    return std::max(longest * alone + once, filled) + (cut > 0 ? 3.2 + cut * 0.29e-6 : 0);
}

// The host takes 0.07 us a work for it: 1.6 us of a call of one matrix, 77 of one of 72, 5 a launch.
Cut choose_cut(const NsWorks &t, size_t room) {
    Cut best = {};
    double cost = 0;
    for (uint32_t edge : {128u, 64u})
        for (uint32_t most : {1u << 30, 256u, 128u, 64u, 32u, 16u, 8u}) {
            const double c = cost_of(t, {edge, most}, room);
            if (c >= 0 && (best.edge == 0 || c < cost)) {
                cost = c;
                best = {edge, most};
            }
        }
    return best;
}

// The works of a batch's launch `k`; those with the longest sums first.
void works_of(const Batch &b, const Program p[2], uint32_t k, NsWorks &t) {
    t.n = 0;
    for (uint32_t m = 0; m < b.t.n; m++) {
        const Program &q = p[b.blocked_[m]];
        for (uint32_t i = 0; i < 2 && k < q.n; i++)
            if (q.op[k][i] != ~0u) {
                t.w[t.n] = b.w[m];
                t.w[t.n++].op |= q.op[k][i];
            }
    }
    std::sort(t.w, t.w + t.n, [](const NsWork &x, const NsWork &y) { return panels_of(x) > panels_of(y); });
    t.mixed = t.n > 1 && panels_of(t.w[0]) != panels_of(t.w[t.n - 1]);
}

// Sets every work's pieces and first item: the launch's items, and the tiles that are cut.
struct Items {
    uint32_t all, cut_tiles;
};
Items cut_works(NsWorks &t, Cut c) {
    Items n = {};
    for (uint32_t k = 0; k < t.n; k++) {
        NsWork &w = t.w[k];
        const uint32_t tiles = tiles_of(w, c.edge);
        w.pieces = pieces_of(panels_of(w), c.most);
        w.begin = n.all;
        n.all += tiles * w.pieces;
        if (w.pieces > 1) n.cut_tiles += tiles;
    }
    return n;
}

// Whether a batch takes the narrow path, a launch per step: every shorter side at
// most 128, few enough turns per workgroup, no more workgroups than the GPU takes at once.  Sets up
// the works, the workgroups and the widest matrix.  Narrow against the products' path, us:
// 64 x 64 47 / 79, 64 x 1024 (one turn) 60 / 113, 64 x 4096 (four) 93 / 114, 64 x 8192 (eight) 134 / 122; 128 x 128
// 79 to 82 / 91, 128 x 1024 (two) 103 to 107 / 112, eight of them 116 to 122 / 123, 32 168 to 176 / 182, 128 x 2048 (four) 137 / 115
// (the larger of two: fp32, with a fourth product).
struct Narrow {
    NsWorks t;
    uint32_t groups, widest;
    uint64_t floats() const { return (uint64_t)groups * narrow_part(widest); }  // of one set of parts
};
bool narrow(const Batch &b, Narrow &n) {
    n.groups = n.widest = 0;
    n.t.n = b.t.n;
    for (uint32_t k = 0; k < b.t.n; k++) {
        NsWork &w = n.t.w[k] = b.w[k];
        const uint32_t S = padded(std::min(w.rows, w.cols)), L = padded(std::max(w.rows, w.cols));
        if (S > kNarrowShort) return false;
        const uint32_t tiles = L / kNarrowCols, most = S == 64 ? 16 : 8, subs = blocks(tiles, most);
        if (subs > (S == 64 ? 4u : 2u)) return false;
        w.pieces = blocks(tiles, subs);
        w.op |= subs << 20;
        w.begin = n.groups;
        n.groups += w.pieces;
        n.widest = std::max(n.widest, S);
    }
    return n.groups <= kNarrowMost && 2 * n.floats() * sizeof(float) <= b.piece_bytes();
}

// The steps on a batch.  src: where the matrices come from; out: where the
// results go (a dtype, or kNsMuonF32).
int run_batch(Batch &b, const Program p[2], uint32_t steps, int src, int out, NsArgs a, void *ws, hipStream_t s) {
    a.ws = (char *)ws;
    a.part = (double *)((char *)ws + b.regions);
    a.pieces = (float *)((char *)ws + b.regions + b.part_bytes());
    uint32_t g = b.spread([&](const NsMat &m) { return b.sums(m); });
    hipError_t e = timed(b.muon ? K_MUON_SUM : K_NS_SUM, s, [&] { return launch_ns_sum(src, b.t, a, g, s); });
    if (e != hipSuccess) return hip_fail(e, "norm launch");
    g = b.spread([&](const NsMat &m) { return blocks(m.rows, kNsPad) * blocks(m.cols, kNsPad); });
    e = timed(K_NS_PREPARE, s, [&] { return launch_ns_prepare(src, b.t, a, g, s); });
    if (e != hipSuccess) return hip_fail(e, "prepare launch");
    Narrow n;
    if (narrow(b, n)) {
        // the parts of A go to one half of the room for pieces and come from the other
        for (uint32_t k = 0; k <= steps; k++) {
            float *to = a.pieces + (k % 2) * n.floats(), *from = a.pieces + (1 - k % 2) * n.floats();
            e = timed(K_NS_NARROW, s, [&] {
                return launch_ns_narrow(out, n.t, a, from, to, k == 0, k == steps, n.groups, n.widest, s);
            });
            if (e != hipSuccess) return hip_fail(e, "narrow step launch");
        }
        return DEDLOC_OK;
    }
    NsWorks t;
    for (uint32_t k = 0; k < std::max(p[0].n, p[1].n); k++) {
        works_of(b, p, k, t);
        if (t.n == 0) break;
        const Cut c = choose_cut(t, b.piece_bytes());
        const Items n = cut_works(t, c);
        e = timed(K_NS_PRODUCT, s, [&] { return launch_ns_product(out, c.edge, t, a, n.all, s); });
        if (e != hipSuccess) return hip_fail(e, "product launch");
        if (n.cut_tiles == 0) continue;
        e = timed(K_NS_JOIN, s, [&] { return launch_ns_join(out, c.edge, t, a, n.cut_tiles, s); });
        if (e != hipSuccess) return hip_fail(e, "join launch");
    }
    return DEDLOC_OK;
}

// Calls run(batch) on the matrices of a call in batches.  next(k, batch) adds
// matrix k; sides(k, rows, cols) gives its sides.
template <typename S, typename N, typename R>
int in_batches(bool muon, bool fp32, uint32_t n, S sides, N next, R run) {
    Batch b(muon, fp32);
    for (uint32_t k = 0; k < n; k++) {
        uint32_t rows = 0, cols = 0;
        sides(k, rows, cols);
        if (rows == 0 || cols == 0) continue;
        if (!b.fits(rows, cols)) {
            const int rc = run(b);
            if (rc) return rc;
            b.clear();
        }
        next(k, b);
    }
    return b.t.n ? run(b) : DEDLOC_OK;
}

int check_ws(const void *ws, size_t have, size_t need) {
    if (!ws || have < need)
        return fail(DEDLOC_ERR_WORKSPACE, "workspace of %zu bytes needed (got %zu)", need, ws ? have : (size_t)0);
    if (!aligned(ws, 256)) return fail(DEDLOC_ERR_ALIGN, "workspace must be 256-byte aligned");
    return DEDLOC_OK;
}

// Workspace of matrices given by their sides: the largest batch's, for results of any type.
template <typename S>
size_t batches_bytes(bool muon, uint32_t n, S sides) {
    for (uint32_t k = 0; k < n; k++) {
        uint32_t rows = 0, cols = 0;
        sides(k, rows, cols);
        if (check_sides(k, rows, cols)) return 0;
    }
    size_t most = 256;
    for (bool fp32 : {false, true}) {
        if (muon && fp32) break;
        in_batches(muon, fp32, n, sides,
                   [&](uint32_t k, Batch &b) {
                       uint32_t rows = 0, cols = 0;
                       sides(k, rows, cols);
                       b.add(nullptr, 0, nullptr, 0, rows, cols, 0, 0.0f);
                   },
                   [&](Batch &b) {
                       most = std::max(most, b.bytes());
                       return DEDLOC_OK;
                   });
    }
    return most;
}

// ------------------------------------------------ embedding and its gradient

struct EmbedWs {
    size_t pairs, counts, total;
    uint32_t chunk, run;
};
// The chunks of a call get shorter below three products of positions and width, so that fewer positions may leave
// more parts: the workspace has room for every smaller call on it, of fewer positions, narrower rows or both.
EmbedWs embed_ws(uint64_t n, uint32_t width) {
    EmbedWs w;
    w.pairs = round_up((size_t)n * sizeof(uint2), 256);
    const uint32_t tiles = std::max(1u, blocks(n, kSortTile));
    w.chunk = (tiles + kSortChunks - 1) / kSortChunks * kSortTile;
    w.counts = ((size_t)std::min(tiles, kSortChunks) << kSortBits) * sizeof(uint32_t);
    // Short chunks where there is little to sum, long ones where the parts of cut runs are many.  4, 8, 16, 32 positions, us: 1000 x
    // 512 14, 16, 21, 29; 8192 x 128 22.9, 22.2, 24.5, 30; 8192 x 768 28.7, 27.3, 30.3, 39; 40000 x 333 88, 81, 76, 95; 65536 x 1024
    // 147, 102, 84, 75.
    struct {
        uint32_t run;
        uint64_t below;
    } const rules[] = {{4, 1u << 20}, {8, 1u << 23}, {16, 1u << 25}, {32, ~0ull}};
    const uint64_t all = n * width;
    uint64_t most = 0;  // whole chunks times their width, of the calls that fit
    for (const auto &r : rules) {
        w.run = r.run;
        most = std::max(most, std::min(all, r.below) / r.run);
        if (all < r.below) break;
    }
    w.total = 2 * w.pairs + w.counts + round_up((size_t)(most + width) * 2 * sizeof(float), 256);  // and a part of a chunk
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
    Program p[2];
    make_program(*cfg, false, p[0]);
    make_program(*cfg, true, p[1]);
    NsArgs a = {};
    a.a = cfg->a;
    a.b = cfg->b;
    a.c = cfg->c;
    a.eps = cfg->eps;
    return in_batches(
        false, dtype == DEDLOC_DTYPE_F32, n,
        [&](uint32_t k, uint32_t &rows, uint32_t &cols) {
            rows = mats[k].rows;
            cols = mats[k].cols;
        },
        [&](uint32_t k, Batch &b) {
            const dedloc_matrix &m = mats[k];
            b.add(m.in, m.ld_in, m.out, m.ld_out, m.rows, m.cols, 0, 0.0f);
        },
        [&](Batch &b) { return run_batch(b, p, cfg->steps, dtype, dtype, a, ws, (hipStream_t)stream); });
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
    Program p[2];
    make_program(cfg->ortho, false, p[0]);
    make_program(cfg->ortho, true, p[1]);
    NsArgs a = {};
    a.a = cfg->ortho.a;
    a.b = cfg->ortho.b;
    a.c = cfg->ortho.c;
    a.eps = cfg->ortho.eps;
    a.x = x;
    a.mom = m;
    a.grad = grad;
    a.scales = grad_scales;
    a.mu = cfg->momentum;
    a.keep = (float)(1.0 - (double)cfg->lr * (double)cfg->weight_decay);
    a.nesterov = cfg->nesterov;
    return in_batches(
        true, false, n_tensors,
        [&](uint32_t k, uint32_t &r, uint32_t &c) {
            r = rows[k];
            c = cols[k];
        },
        [&](uint32_t k, Batch &b) {
            const double ratio =
                flags[k] & DEDLOC_TENSOR_ADAPT ? (double)cfg->rms * sqrt((double)std::max(rows[k], cols[k])) : 1.0;
            b.add(nullptr, offsets[k], nullptr, offsets[k], rows[k], cols[k], flags[k], (float)((double)cfg->lr * ratio));
        },
        [&](Batch &b) { return run_batch(b, p, cfg->ortho.steps, src, kNsMuonF32, a, ws, (hipStream_t)stream); });
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
                             scale * batch_samples, w.chunk, w.run, {(uint2 *)b, (uint2 *)(b + w.pairs)}, (uint32_t *)(b + 2 * w.pairs),
                             (float *)(b + 2 * w.pairs + w.counts)};
    hipStream_t s = (hipStream_t)stream;
    int from = -1;
    if (n <= kSortOne) {
        hipError_t e = timed(K_EMBED_SORT, s, [&] { return launch_embed_sort(a, s); });
        if (e != hipSuccess) return hip_fail(e, "embed sort launch");
        from = 0;
        if (n > 1024) {
            e = timed(K_EMBED_MERGE, s, [&] { return launch_embed_merge(a, s); });
            if (e != hipSuccess) return hip_fail(e, "embed merge launch");
            from = 1;
        }
    }
    if (n > kSortOne) {
        // as few digits as hold the tokens and `vocab`, which stands for a masked position
        uint32_t all = 1;
        while (vocab >> all) all++;
        const uint32_t passes = (all + kSortBits - 1) / kSortBits, bits = std::max(8u, (all + passes - 1) / passes);
        for (uint32_t shift = 0; shift < all; shift += bits) {
            hipError_t e = timed(K_EMBED_COUNT, s, [&] { return launch_embed_count(a, from, bits, shift, s); });
            if (e != hipSuccess) return hip_fail(e, "embed count launch");
            e = timed(K_EMBED_SCATTER, s, [&] { return launch_embed_scatter(a, from, bits, shift, s); });
            if (e != hipSuccess) return hip_fail(e, "embed scatter launch");
            from = from < 0 ? 0 : 1 - from;
        }
    }
    hipError_t e = timed(K_EMBED_SUM, s, [&] { return launch_embed_sum(dy_dtype, a, from, s); });
    if (e != hipSuccess) return hip_fail(e, "embed sum launch");
    e = timed(K_EMBED_JOIN, s, [&] { return launch_embed_join(a, from, s); });
    return e == hipSuccess ? DEDLOC_OK : hip_fail(e, "embed join launch");
}

}  // extern "C"
