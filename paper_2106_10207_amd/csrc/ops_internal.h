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

// A launch describes at most kNsMats matrices in its arguments (56 of 64
// bytes: 3.5 KB of the 4 KB that kernel arguments may take).
constexpr int kNsMats = 56;
constexpr uint32_t kNsPad = 64;      // both sides of a matrix are padded with zeros to this in the workspace
constexpr uint32_t kNsTile = 64;     // edge of a block of the elementwise passes
constexpr uint32_t kNsMaxShort = 32768;
constexpr uint32_t kNsMaxLong = 1u << 26;
constexpr uint32_t kSumChunk = 8192;  // flat elements summed by one workgroup of the momentum pass

// One matrix of a launch.  s is its shorter side, l the longer; S and L are s
// and l rounded up to kNsPad.  Its region of the workspace, at `base` bytes:
//   X [S][L], X^T [L][S] twice (read and written in turn), A [S][S], B [S][S]
// in two planes (4 bytes an element).
struct NsMat {
    uint64_t base;
    const void *in;         // orthogonalize: the matrix
    void *out;
    uint64_t ld_in, ld_out;  // Muon: ld_in is the matrix' first element in the flat vector
    uint32_t rows, cols;
    uint32_t part;          // its first partial sum; the next matrix' is the end
    uint32_t begin;         // its first workgroup in this launch
    uint32_t flags;
    float unit;             // Muon: lr * s_t
};
struct NsTable {
    NsMat m[kNsMats];
    uint32_t n;
    uint32_t parts;  // partial sums of all matrices
};

struct NsArgs {
    char *ws;        // the regions
    double *part;    // partial sums of squares
    float *x, *mom;  // Muon: the flat vector and the momentum
    const void *grad;
    const float *scales;
    float a, b, c, eps;
    float mu, keep;  // momentum; 1 - lr * weight_decay
    int32_t nesterov;
    int32_t turn;    // which X^T is read (the other is written)
    int32_t last;    // the last step: the result goes out instead of into the workspace
};

// Where prepare takes its matrix from: a dtype of orthogonalize, or the Muon
// step's update formed from the momentum and a gradient of this codec.
enum NsSrc : int { kNsF32 = 0, kNsFP16 = 1, kNsBF16 = 2, kNsMuonF32 = 3, kNsMuonFP16 = 4, kNsMuonI8 = 5 };
enum NsPhase : int { kNsGram = 0, kNsSquare = 1, kNsApply = 2 };

hipError_t launch_ns_sum(int src, const NsTable &t, const NsArgs &a, uint32_t groups, hipStream_t s);
hipError_t launch_ns_prepare(int src, const NsTable &t, const NsArgs &a, uint32_t groups, hipStream_t s);
hipError_t launch_ns_product(int phase, int out, bool wide, const NsTable &t, const NsArgs &a, uint32_t groups, hipStream_t s);

// ------------------------------------------------ embedding and its gradient

constexpr uint32_t kEmbedMaxTokens = 1u << 30;
constexpr uint32_t kEmbedMaxVocab = 1u << 30;
constexpr uint32_t kEmbedMaxWidth = 1u << 20;
// Positions are sorted in at most kSortChunks chunks of whole tiles, one
// workgroup each: every workgroup reads the digit counts of all chunks.
constexpr uint32_t kSortTile = 2048;
constexpr uint32_t kSortChunks = 512;
constexpr uint32_t kRunChunk = 32;     // sorted positions summed by one row of threads

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
    // workspace: (token, position) pairs sorted in turn between two buffers,
    // digit counts per chunk, and the sums of runs cut by a chunk's edge
    uint2 *pairs[2];
    uint32_t *counts;
    float *cut;  // [chunks][2][width]
};

hipError_t launch_embed(int table, int out, const EmbedArgs &a, hipStream_t s);
hipError_t launch_embed_count(const EmbedGradArgs &a, int from, uint32_t shift, hipStream_t s);
hipError_t launch_embed_scatter(const EmbedGradArgs &a, int from, uint32_t shift, hipStream_t s);
hipError_t launch_embed_sum(int dy, const EmbedGradArgs &a, int sorted, hipStream_t s);
hipError_t launch_embed_join(const EmbedGradArgs &a, int sorted, hipStream_t s);

}  // namespace dedloc
