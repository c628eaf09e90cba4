// gfx950 kernel of norms of rows and of the end of one block with the start of the
// next in one pass (the branch's norm, gate, dropout, the residual sum and its
// norm).  Bound by the bytes of the rows: a row is read once, held in
// registers by the threads that share it, and written once.
#pragma once

#include <algorithm>

#include "block_rows.h"

namespace dedloc {

// The teams of a launch take the rows in turn; a row's vectors are on their way while the one before is worked on.  What a
// thread's columns are scaled by stays in its registers.  MODE 0: the norm of h; 1: a branch without a post norm; 2: with one; 3: with
// a gate per group of rows.  Bound by memory: 65536 x 2048 fp32 with bf16 branches, two norms, a gate and dropout 295 us, 5.5 TB/s
// (vector instructions in 0.4 of the cycles); 65536 x 1024 bf16 with one norm and dropout 96 us, 5.6 TB/s; the rms norm of 65536 x
// 2048 bf16 89 us, 6.0 TB/s.  8192 x 1024 fp16 12.5 us: three rows a team, ramp and end.
template <typename TS, typename TB, int T, int V, int MOST, int MODE, bool STREAM, bool RAGGED>
__global__ __launch_bounds__(MOST, resident(kForwardWaves, V, MODE, MOST)) void residual_kernel(ResidualArgs a, uint32_t waves, uint32_t all) {
    constexpr int N = V * E;
    __shared__ Meet<MOST> meet;
    constexpr bool SPLIT = sizeof(TS) == 4;
    const Team<T, V, MOST, SPLIT, RAGGED> team(waves, a.width, &meet);
    uint32_t row = T < 64 ? (blockIdx.x * MOST + threadIdx.x) / T : blockIdx.x;
    if (T == 64 && waves == 1) row = blockIdx.x * (MOST / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    // v = times * fhat + plus, and pre's gain and bias
    float times[N], plus[N], gain[N], bias[N];
    Mask mask[V];
    const bool shared = MODE > 0 && MODE < 3 && a.gate;
#pragma unroll
    for (int v = 0; v < V; v++) {
        team.parameters(a.pre.gain, v, 1.0f, gain + v * E);
        team.parameters(a.pre.bias, v, 0.0f, bias + v * E);
        if constexpr (MODE > 1) {
            team.parameters(a.post.gain, v, 1.0f, times + v * E);
            team.parameters(a.post.bias, v, 0.0f, plus + v * E);
        }
        if constexpr (MODE > 0) {
            float g[E];
            team.parameters(shared ? (const float *)a.gate : nullptr, v, 1.0f, g);
#pragma unroll
            for (int i = 0; i < E; i++) {
                times[v * E + i] = MODE > 1 ? times[v * E + i] * g[i] : g[i];
                if (MODE > 1) plus[v * E + i] *= g[i];
            }
            if (a.drop.threshold) mask[v].init(a.drop, step_of(a.drop), team.counter(v));
        }
    }
    Raw<TS> h[V], next_h[V] = {};
    Raw<TB> f[V], next_f[V] = {}, gate[V], next_gate[V] = {};
    const auto fetch = [&](uint32_t r) {
        const TS *from = (const TS *)a.h + r * a.ld_h;
        const TB *from_f = (const TB *)a.f + r * a.ld_f, *from_gate = nullptr;
        if constexpr (MODE == 3) from_gate = (const TB *)a.gate + r / a.gate_rows * a.ld_gate;
#pragma unroll
        for (int v = 0; v < V; v++) {
            // zeros into registers of their own: what is on its way need not arrive first
            next_h[v] = {};
            next_f[v] = next_gate[v] = {};
            team.pieces(v, [&](int p) {
                team.template load<STREAM>(next_h[v], from, v, p);
                if constexpr (MODE > 0) team.template load<STREAM>(next_f[v], from_f, v, p);
                if constexpr (MODE == 3) team.template load<false>(next_gate[v], from_gate, v, p);
            });
        }
    };
    // Loads and stores are counted as one: a wait for the next row's loads would be one for this row's stores too, of which some may
    // have been left out, so the loads have to arrive before the last stores begin.
    const auto arrived = [&] {
#pragma unroll
        for (int v = 0; v < V; v++) {
            arrive(next_h[v]);
            if constexpr (MODE > 0) arrive(next_f[v]);
            if constexpr (MODE == 3) arrive(next_gate[v]);
        }
    };
    if (row < a.rows) fetch(row);
    arrived();
    while (row < a.rows) {
#pragma unroll
        for (int v = 0; v < V; v++) {
            h[v] = next_h[v];
            if constexpr (MODE > 0) {
                f[v] = next_f[v];
                if constexpr (MODE == 3) gate[v] = next_gate[v];
            }
        }
        const uint32_t at = row;
        row += all;
        if (row < a.rows) fetch(row);
        float x[N];
#pragma unroll
        for (int v = 0; v < V; v++) team.unpack(h[v], v, x + v * E);
        if constexpr (MODE > 0) {
            float y[N];
#pragma unroll
            for (int v = 0; v < V; v++) team.unpack(f[v], v, y + v * E);
            float2 st = make_float2(0.0f, 1.0f);
            if (MODE == 2 || (MODE == 3 && a.post.kind)) {
                st = team.template stats<TB>(y, a.post);
                if (a.stats && team.t == 0) a.stats[a.rows + at] = st;
            }
            if (!a.pre.kind) arrived();
#pragma unroll
            for (int v = 0; v < V; v++) {
                float *z = y + v * E;
#pragma unroll
                for (int i = 0; i < E; i++)
                    z[i] = MODE > 1 ? fmaf((z[i] - team.about(v, i, st.x)) * st.y, times[v * E + i], plus[v * E + i]) : z[i] * times[v * E + i];
                if constexpr (MODE == 3) {
                    float g[E];
                    team.unpack(gate[v], v, g);
#pragma unroll
                    for (int i = 0; i < E; i++) z[i] *= g[i];
                }
                if (a.drop.threshold) mask[v].template apply<SPLIT>(a.drop, at, a.drop.factor, z);
#pragma unroll
                for (int i = 0; i < E; i++)  // the norm sees the sum as it is stored
                    x[v * E + i] = rounded<TS>(fmaf(a.beta, z[i], a.alpha * x[v * E + i]));
                if (a.sum) team.pieces(v, [&](int p) { team.template store<true>((TS *)a.sum + at * a.ld_sum, v, p, x + v * E); });
            }
        }
        if (!a.pre.kind) continue;
        const float2 st = team.template stats<TS>(x, a.pre);
        arrived();
        if (a.stats && team.t == 0) a.stats[at] = st;
#pragma unroll
        for (int v = 0; v < V; v++) {
#pragma unroll
            for (int i = v * E; i < (v + 1) * E; i++) x[i] = fmaf((x[i] - st.x) * st.y, gain[i], bias[i]);
            team.pieces(v, [&](int p) { team.template store<true>((TB *)a.out + at * a.ld_out, v, p, x + v * E); });
        }
    }
}

template <typename TS, typename TB>
void launch_forward(const ResidualArgs &a, hipStream_t s) {
    const RowShape r = forward_shape(a.width, sizeof(TS) == 4);
    const int mode = forward_mode(a);
    const uint32_t most = kSimds * resident(kForwardWaves, r.vectors, mode, r.threads) * 64 / r.threads;
    const uint32_t groups = std::min((a.rows + r.teams() - 1) / r.teams(), most);
    const bool stream = (uint64_t)a.rows * a.width * (sizeof(TS) + (a.f ? sizeof(TB) : 0)) >= kStreamBytes;
    with_shape(r, [&](auto sh) {
        with_mode(mode, [&](auto m) {
            typedef decltype(sh) S;
            with_access<S>(ragged_row(a.width, sizeof(TS) == 4), stream, [&](auto streaming, auto ragged) {
                residual_kernel<TS, TB, S::T, S::V, S::MOST, decltype(m)::value, decltype(streaming)::value, decltype(ragged)::value>
                    <<<groups, r.threads, 0, s>>>(a, r.waves(), groups * r.teams());
            });
        });
    });
}

}  // namespace dedloc
