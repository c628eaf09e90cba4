// Internal declarations of the model-step operators (orthogonalised updates,
// the Muon step, the embedding lookup and its gradient) shared by their
// kernels and their C-ABI layer.  Not part of the public interface.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dedloc {

// ---------------------------------------------------- orthogonalised updates

// Element types, as the DEDLOC_DTYPE_* ids.
enum Dtype : int { kF32 = 0, kFP16 = 1, kBF16 = 2 };

// A launch describes at most kNsWorks products in its arguments (48 bytes each,
// 3.4 KB of the 4 KB that kernel arguments may take).
constexpr int kNsWorks = 72;
constexpr uint32_t kNsPad = 64;   // both sides of a matrix are padded with zeros to this in the workspace
constexpr uint32_t kNsTile = 64;  // edge of a block of the elementwise passes
constexpr uint32_t kNsMaxShort = 32768;
constexpr uint32_t kNsMaxLong = 1u << 26;
constexpr uint32_t kSumChunk = 8192;  // flat elements that a workgroup of the momentum pass sums at a time
// Sums of squares of a matrix at most: every workgroup of the next pass adds them all up, 8 a thread.
constexpr uint32_t kSumMost = 2048;

// A matrix has a region of the workspace.  s is its shorter side, l the longer; S
// and L are s and l rounded up to kNsPad.  The region holds, 4 bytes an element,
//   buffer 0: X [S][L],  1 and 2: X^T [L][S], read and written in turn,
//   buffers 3 on: symmetric [S][S].
constexpr uint32_t kNsSmall = 3;   // the first symmetric buffer
constexpr uint32_t kNsSmalls = 6;  // of a matrix that is worked on in blocks of steps; 2 otherwise

// The two passes before the products.
struct NsMat {
    uint64_t base;     // its region
    const void *in;    // orthogonalize: the matrix
    uint64_t ld_in;    // Muon: its first element in the flat vector
    uint32_t rows, cols;
    uint32_t part;     // its first partial sum; the next matrix' is the end
    uint32_t begin;    // its first workgroup in this launch
};
// A table's arguments are copied at every launch: 3.5 KB take the host 4.1 us, 0.4 KB 2.6.
constexpr int kNsFew = 8;
template <int N>
struct NsMats {
    NsMat m[N];
    uint32_t n;
    uint32_t parts;  // partial sums of all matrices
};
typedef NsMats<kNsWorks> NsTable;

// One product of a launch, left right^T, and what becomes of it:
enum NsKind : int {
    kNsGram = 0,    // X X^T, symmetric
    kNsSquare = 1,  // a I + b A + c A A, symmetric
    kNsMul = 2,     // of two commuting symmetric matrices
    kNsApply = 3,   // Q X: the next X and X^T
    kNsResult = 4   // Q X: the call's result
};
struct NsWork {
    uint64_t base;
    void *out;        // kNsResult: orthogonalize's matrix
    uint64_t ld_out;  // Muon: its first element in the flat vector
    uint32_t rows, cols;
    uint32_t begin;   // its first work item in this launch
    uint32_t pieces;  // that the summed index is cut into
    uint32_t op;      // kind | left << 4 | right << 8 | out << 12 (buffers) | decay << 16; narrow: turns << 20
    float unit;       // Muon: lr * s_t
};
template <int N>
struct NsList {
    NsWork w[N];
    uint32_t n;
    uint32_t mixed;  // products: whether their summed indexes differ in length
};
typedef NsList<kNsWorks> NsWorks;

struct NsArgs {
    char *ws;        // the regions
    double *part;    // partial sums of squares
    float *pieces;   // sums of the items whose summed index is cut, a tile each
    float *x, *mom;  // Muon: the flat vector and the momentum
    const void *grad;
    const float *scales;
    float a, b, c, eps;
    float mu, keep;  // momentum; 1 - lr * weight_decay
    int32_t nesterov;
};

// Narrow matrices: a workgroup owns kNarrowCols columns of X and, of a long matrix,
// as many more times as leave at most 16 workgroups (8 with a side of 128; each adds up
// every part of A: 16 KB of a side of 64, 64 KB less the upper triangle of 128).
constexpr uint32_t kNarrowShort = 128;
constexpr uint32_t kNarrowCols = 64;

// Where prepare takes its matrix from: a dtype of orthogonalize, or the Muon
// step's update formed from the momentum and a gradient of this codec.
enum NsSrc : int { kNsF32 = 0, kNsFP16 = 1, kNsBF16 = 2, kNsMuonF32 = 3, kNsMuonFP16 = 4, kNsMuonI8 = 5 };

hipError_t launch_ns_sum(int src, const NsTable &t, const NsArgs &a, uint32_t groups, hipStream_t s);
hipError_t launch_ns_prepare(int src, const NsTable &t, const NsArgs &a, uint32_t groups, hipStream_t s);
// out: the dtype of results, kNsMuonF32 for the update of the parameters.  edge: of
// the tiles, 64 or 128.  The works whose summed index is cut come first in the
// table; join takes their number of tiles.
hipError_t launch_ns_product(int out, uint32_t edge, const NsWorks &t, const NsArgs &a, uint32_t items, hipStream_t s);
hipError_t launch_ns_join(int out, uint32_t edge, const NsWorks &t, const NsArgs &a, uint32_t tiles, hipStream_t s);

// A step of narrow matrices.  widest: the largest S among them; the parts of A, one of narrow_part(widest) floats per
// workgroup, are read from `from` and left in `to`.
inline uint32_t narrow_part(uint32_t widest) { return (widest / 32) * (widest / 32 + 1) / 2 * 1024; }
hipError_t launch_ns_narrow(int out, const NsWorks &t, const NsArgs &a, const float *from, float *to, bool first, bool last,
                            uint32_t groups, uint32_t widest, hipStream_t s);

// ------------------------------------------------ embedding and its gradient

constexpr uint32_t kEmbedMaxTokens = 1u << 30;
constexpr uint32_t kEmbedMaxVocab = 1u << 30;
constexpr uint32_t kEmbedMaxWidth = 1u << 20;
// Positions are sorted in at most kSortChunks chunks of whole tiles, one
// workgroup each: every workgroup reads the digit counts of all chunks.
constexpr uint32_t kSortTile = 2048;
constexpr uint32_t kSortChunks = 512;
constexpr uint32_t kSortBits = 10;  // of a digit at most
// Up to kSortOne positions are sorted in chunks of 1024 and merged.
constexpr uint32_t kSortOne = 16384;

struct EmbedArgs {
    const void *table;
    uint64_t ld_table;
    const void *ids;
    void *out;
    uint64_t ld_out;
    uint32_t vocab, width, n;
    int32_t wide_ids;  // 64-bit ids
    float scale;
};

struct EmbedGradArgs {
    float *grad;
    uint64_t ld_grad;
    const void *ids;
    const void *dy;
    uint64_t ld_dy;
    uint32_t vocab, width, n;
    int32_t wide_ids;
    float factor;    // scale * batch_samples
    uint32_t chunk;  // positions of a chunk of the sort
    uint32_t run;    // sorted positions summed by one row of threads
    // workspace: (token, position) pairs sorted in turn between two buffers,
    // digit counts per chunk, and the sums of runs cut by a chunk's edge
    uint2 *pairs[2];
    uint32_t *counts;
    float *cut;  // [chunks][2][width]
};

hipError_t launch_embed(int table, int out, const EmbedArgs &a, hipStream_t s);
// The sort of at most kSortOne positions: chunks of 1024 into pairs[0], merged into pairs[1].
hipError_t launch_embed_sort(const EmbedGradArgs &a, hipStream_t s);
hipError_t launch_embed_merge(const EmbedGradArgs &a, hipStream_t s);
// One pass over a digit of 8 bits (fewer are taken as 8), 9 or kSortBits; from: the
// buffer that holds the pairs, or -1: the ids.
hipError_t launch_embed_count(const EmbedGradArgs &a, int from, uint32_t bits, uint32_t shift, hipStream_t s);
hipError_t launch_embed_scatter(const EmbedGradArgs &a, int from, uint32_t bits, uint32_t shift, hipStream_t s);
hipError_t launch_embed_sum(int dy, const EmbedGradArgs &a, int sorted, hipStream_t s);
hipError_t launch_embed_join(const EmbedGradArgs &a, int sorted, hipStream_t s);

}  // namespace dedloc
