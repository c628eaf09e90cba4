// Internal declarations of what stands between the matrix products of a model's
// step (dropout, norms, the ends of a block) shared by the kernels and their
// C-ABI layer.  Not part of the public interface.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dedloc {

constexpr uint32_t kBlockMaxRows = 1u << 30;
constexpr uint32_t kDropMaxWidth = 1u << 20;
constexpr uint32_t kNormMaxWidth = 16384;  // a row is held by one workgroup: 1024 threads of 16 columns
constexpr uint32_t kBlockParts = 1024;     // workgroups of a gradient at most: each leaves a part of every vector's gradient
constexpr uint32_t kBlockGrid = 1u << 20;  // workgroups of the other launches at most, of up to 1024 threads
constexpr uint32_t kDropVectors = 2048;    // vectors of a workgroup of the dropout at a time
constexpr uint32_t kBlockSums = 4;         // vectors that the rows are summed into

struct DropArgs {
    uint32_t threshold;  // halves below it drop; 0: no dropout
    float factor;
    uint32_t key0, key1, site, step, row0;
    const int64_t *step_at;  // nullable: added to step
};

enum NormKind : int { kNormNone = 0, kNormLayer = 1, kNormRms = 2 };

struct NormArgs {
    int32_t kind;
    float eps;
    const float *gain, *bias;  // nullable
};

struct DropoutArgs {
    const void *x;
    void *out;
    uint64_t ld_x, ld_out;
    uint32_t rows, width;
    uint32_t per;    // rows of a workgroup
    uint32_t magic;  // ceil(2^32 / vectors of a row)
    DropArgs drop;
};

// stats: (mean, 1 / deviation) of every row's pre norm, then of every row's post norm.
struct ResidualArgs {
    const void *h, *f;  // f NULL: the norm of h alone
    void *sum, *out;    // nullable
    float2 *stats;      // nullable
    uint64_t ld_h, ld_f, ld_sum, ld_out;
    const void *gate;   // nullable
    uint64_t ld_gate;
    uint32_t rows, width, gate_rows;  // gate_rows 0: one fp32 gate for all rows, else one of f's type per gate_rows rows
    float alpha, beta;
    NormArgs post, pre;
    DropArgs drop;
};

struct ResidualGradArgs {
    const void *sum, *f, *dsum, *dout;  // f NULL: the norm of sum alone; dsum, dout nullable
    void *dh, *df;
    const float2 *stats;
    uint64_t ld_sum, ld_f, ld_dsum, ld_dout, ld_dh, ld_df;
    const void *gate;
    uint64_t ld_gate;
    float *dgate;  // nullable
    uint64_t ld_dgate;
    uint32_t rows, width, gate_rows;
    float alpha, beta;
    NormArgs post, pre;
    DropArgs drop;
    float *dpre_gain, *dpre_bias, *dpost_gain, *dpost_bias;  // nullable
    float samples;
    // The rows' sums: 0 dout * xhat, 1 dout of the pre norm; 2 of dv * fhat, 3 of dv of the post norm, dv taken before a
    // gate that all rows share.  want: bit per sum; a workgroup's parts are those sums, one after the other.
    uint32_t want;
    uint32_t groups;  // workgroups
    uint32_t turns;   // rows of a team at most
    int32_t cut;      // a gate per group of rows: a team takes rows that follow each other
    float *part;      // [groups][wanted sums][width]
    float *edge;      // [2][teams][width]: sums of the group of rows at a team's start, and at its end, that its range cuts
};

// How a row is spread over threads: `lanes` of them, 8 columns of a vector each, `vectors` times over.
struct RowShape {
    uint32_t lanes;    // 8, 16, 32 or 64 times the waves of a row
    uint32_t vectors;  // 1 or 2
    uint32_t threads;  // of a workgroup
    uint32_t teams() const { return threads / lanes; }
};
RowShape row_shape(uint32_t width);

hipError_t launch_dropout(int dtype, const DropoutArgs &a, hipStream_t s);
hipError_t launch_residual(int stream, int branch, const ResidualArgs &a, hipStream_t s);
hipError_t launch_residual_grad(int stream, int branch, const ResidualGradArgs &a, hipStream_t s);
hipError_t launch_residual_join(const ResidualGradArgs &a, hipStream_t s);
hipError_t launch_gate_join(const ResidualGradArgs &a, hipStream_t s);

}  // namespace dedloc
