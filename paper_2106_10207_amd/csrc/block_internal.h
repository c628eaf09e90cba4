// Internal declarations of what stands between the matrix products of a model's
// step (dropout, norms, the ends of a block) shared by the kernels and their
// C-ABI layer.  Not part of the public interface.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "ops_internal.h"

namespace dedloc {

constexpr uint32_t kBlockMaxRows = 1u << 30;
constexpr uint32_t kDropMaxWidth = 1u << 20;
constexpr uint32_t kNormMaxWidth = 16384;  // a row is held by one workgroup: 1024 threads of 16 columns
constexpr uint32_t kBlockGrid = 1u << 20;  // workgroups of a launch at most
constexpr uint32_t kDropThreads = 512;     // of a workgroup of the dropout at most
constexpr uint32_t kDropBatch = 4;         // rows of a thread of it that are loaded at a time
constexpr uint32_t kDropGroups = 4096;     // its workgroups at least before a thread takes more rows
// Calls whose inputs take more read them past the caches: less is likely to be there still from the kernel that wrote it.  Through
// and past them: norm_grad of 67 MB 23.7 and 25.8 us, a norm of 67 MB 20.8 and 24.4; dropout of 134 MB 47.8 and 45.9, norm_grad of 201 MB
// 62.9 and 60.0, residual_grad of 1.1 GB 337 and 330.  Results are always written past them (norm_grad of 67 MB 27.5 and 23.6).
constexpr uint64_t kStreamBytes = 96ull << 20;
constexpr uint32_t kBlockSums = 4;         // vectors that the rows are summed into
constexpr uint32_t kSimds = 1024;          // 256 CUs of 4

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
    DropArgs drop;
    // set by the launch
    uint32_t per;           // rows of a workgroup
    uint32_t across, down;  // threads of a row, and rows at a time
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
    int32_t f32;      // the stream's type is fp32
    float *part;      // [groups][wanted sums][width]
    float *edge;      // [2][teams][width]: sums of the group of rows at a team's start, and at its end, that its range cuts
};

// How a row is spread over threads: `lanes` of them, 8 columns of a vector each, `vectors` times over.
struct RowShape {
    uint32_t lanes;    // 8, 16, 32 or 64 times the waves of a row
    uint32_t vectors;  // 1 or 2
    uint32_t threads;  // of a workgroup: whole rows of threads, one where a row takes several waves
    uint32_t waves() const { return lanes / 64; }
    uint32_t teams() const { return threads / lanes; }
};
// columns: of a wave, where a row takes more than a part of one; 512 or 1024
inline RowShape row_shape(uint32_t width, uint32_t columns) {
    if (width <= 64) return {8, 1, 256};
    if (width <= 128) return {16, 1, 256};
    if (width <= 256) return {32, 1, 256};
    const uint32_t few = (width + columns - 1) / columns, waves = few < 16 ? few : 16;
    return {64 * waves, waves * 512 < width ? 2u : 1u, waves == 1 ? 256 : 64 * waves};
}
// Two vectors a thread take fewer meetings of waves and fewer sums over lanes for a row.  They are taken up to 4096 columns, four waves:
// longer rows are compiled for 1024 threads and so for 128 registers, which hold one vector of the forward pass and of a norm's gradient
// alone.  The other gradients of one vector, too, keep up to 68 bytes a thread in scratch, with the sums of a post norm or gate 40 to 232, with groups 208 to 356:
// 32768 x 4096, fp32 stream, 770 us for 412 of its bytes at 5.87 TB/s; 16384 x 8192 bf16 371 for 275.
// 65536 rows of 1024 bf16, one vector and two: residual 101 and 96 us, norm_grad 105 and 94, residual_grad 134 and 122 (8192 columns,
// forward: 185 and 269).  What keeps most in registers stays at one: gates of groups (218 and 362), and fp32 streams with the sums of a
// post norm (65536 x 2048: 468 and 525).
// Ragged rows (see with_access) stay at one too, for the sake of the code's size.
inline bool ragged_row(uint32_t width, bool f32) { return width % (f32 ? 4 : 8); }
inline RowShape forward_shape(uint32_t width, bool f32) { return row_shape(width, width <= 4096 && !ragged_row(width, f32) ? 1024 : 512); }
inline RowShape grad_shape(uint32_t width, int mode, bool f32) {
    return row_shape(width, width <= 4096 && mode < (f32 ? 2 : 3) && !ragged_row(width, f32) ? 1024 : 512);
}

// What a call works on decides the kernel: see the kernels' MODE.
inline int forward_mode(const ResidualArgs &a) { return !a.f ? 0 : a.gate_rows ? 3 : a.post.kind ? 2 : 1; }
inline int grad_mode(const ResidualGradArgs &a) { return !a.df ? 0 : a.gate_rows ? 3 : a.f ? 2 : 1; }
// Waves of a SIMD that the kernels' registers leave room for, by mode and by vectors of a thread.  A launch has that many waves in whole
// workgroups: as many as run at once where a row takes a part of a wave or 1, 2, 4, 8 or 16 of them.  Other numbers of waves leave
// some of a CU's places empty, which this does not count, and the workgroups that do not fit run after the others (gradients of 2560 columns bf16:
// 682 workgroups, 512 at once): residual_grad with one norm 65536 x 2048 5.5 TB/s, 65536 x 2560 3.8; with two and a gate 5.1 and 4.3.
constexpr int kForwardWaves[2][4] = {{6, 5, 4, 4}, {4, 3, 3, 2}}, kGradWaves[2][4] = {{4, 4, 3, 3}, {2, 2, 2, 2}};
constexpr int resident(const int (&waves)[2][4], uint32_t vectors, int mode, uint32_t threads) {
    return threads > 256 ? 4 : waves[vectors - 1][mode];  // 1024 threads leave no less than four
}

// f(a type that names the lanes of a wave that share a row, a thread's vectors and a workgroup's most threads)
template <int T_, int V_, int MOST_>
struct Shape {
    static constexpr int T = T_, V = V_, MOST = MOST_;
};
template <typename F>
void with_shape(const RowShape &r, F f) {
    if (r.lanes == 8) return f(Shape<8, 1, 256>());
    if (r.lanes == 16) return f(Shape<16, 1, 256>());
    if (r.lanes == 32) return f(Shape<32, 1, 256>());
    if (r.threads <= 256 && r.vectors == 1) return f(Shape<64, 1, 256>());
    if (r.threads <= 256) return f(Shape<64, 2, 256>());
    if (r.vectors == 1) return f(Shape<64, 1, 1024>());
    f(Shape<64, 2, 1024>());
}
template <typename F>
void with_mode(int mode, F f) {
    if (mode == 0) return f(std::integral_constant<int, 0>());
    if (mode == 1) return f(std::integral_constant<int, 1>());
    if (mode == 2) return f(std::integral_constant<int, 2>());
    f(std::integral_constant<int, 3>());
}

// f(whether to read past the caches, whether the row's end cuts a piece of the columns that are read at once).  Only rows of
// whole waves are read past the caches, and only those that a thread holds in one vector may be ragged, or in two of more than 8192 columns.
template <typename S, typename F>
void with_access(bool ragged, bool stream, F f) {
    constexpr bool wide = S::V == 2 && S::MOST == 1024;
    if constexpr (S::V == 1 || wide)
        if (ragged) return f(std::false_type(), std::true_type());
    if constexpr (S::T == 64 && !wide)
        if (stream) return f(std::true_type(), std::false_type());
    f(std::false_type(), std::false_type());
}

// The kernels of one pair of types, each in a source file of its own: the stream's type TS, the branch's TB.
template <typename TS, typename TB>
void launch_forward(const ResidualArgs &a, hipStream_t s);
template <typename TS, typename TB>
void launch_grad(const ResidualGradArgs &a, hipStream_t s);

hipError_t launch_dropout(int dtype, DropoutArgs a, hipStream_t s);
hipError_t launch_residual(int stream, int branch, const ResidualArgs &a, hipStream_t s);
hipError_t launch_residual_grad(int stream, int branch, const ResidualGradArgs &a, hipStream_t s);
hipError_t launch_residual_join(const ResidualGradArgs &a, hipStream_t s);
hipError_t launch_gate_join(const ResidualGradArgs &a, hipStream_t s);

}  // namespace dedloc
