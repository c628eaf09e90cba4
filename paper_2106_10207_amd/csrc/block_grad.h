// gfx950 kernel of the gradients of norms of rows and of the ends of a block
// (block_forward.h).  A row's gradient needs the row alone; the gradients of the
// vectors that scale all rows are sums over the rows, which every workgroup
// keeps in registers and leaves as parts, joined (block.hip) in an order fixed by the sizes.
#pragma once

#include "block_rows.h"

namespace dedloc {

// MODE 0: the norm of the sum alone; 1: a branch whose values are not needed (no post norm, no gradient of a gate); 2: with the sums of
// its norm or gate; 3: and a gate per group of rows.
// The formulas, with x the sum and f the branch, xhat = (x - mean) r, fhat likewise with r', g = gain dout:
//   d = dsum + r (g - mean(g) - xhat mean(g xhat)),  dh = alpha d,  w = beta dropout(d)
//   p = times w (times: gate and post's gain),  df = r' (p - mean(p) - fhat mean(p fhat))
// Rows are taken as in the forward pass.  Bound by memory, with vector instructions in half of the cycles: 65536 x 2048 bf16 with
// two norms, a gate and dropout 304 us, 5.3 TB/s; 65536 x 1024 with one norm and dropout 123 with the join, 5.4 TB/s; an fp32 stream
// of 65536 x 2048 445, 5.4 TB/s; 262144 x 64 bf16 18 us.  8192 x 1024 fp16 15 us: four rows a team.  Past 8192 columns two vectors
// do not fit 128 registers, up to 764 bytes a thread lie in scratch: 8192 x 16384 bf16 with one norm 419 us, 2.6 TB/s, with two
// and a gate 1003.  Gates of groups do not fit their 168 registers either (12 to 80 bytes of scratch in 16 bits, 80 to 232 in fp32): 65536 x 1024
// with a gate per 512 rows 197 to 204 us, 4.0 TB/s.
template <typename TS, typename TB, int T, int V, int MOST, int MODE, bool STREAM, bool RAGGED>
__global__ __launch_bounds__(MOST, resident(kGradWaves, V, MODE, MOST)) void residual_grad_kernel(ResidualGradArgs a, uint32_t waves,
                                                                                                  uint32_t all) {
    constexpr int N = V * E;
    constexpr bool BRANCH = MODE > 0, SUMS = MODE > 1, GROUPS = MODE > 2;
    __shared__ Meet<MOST> meet;
    __shared__ float cells[T < 64 ? 4 * T * E : MOST == 256 ? 4 * 64 * N : 1];
    constexpr bool SPLIT = sizeof(TS) == 4;
    const Team<T, V, MOST, SPLIT, RAGGED> team(waves, a.width, &meet);
    uint32_t id = T < 64 ? (blockIdx.x * MOST + threadIdx.x) / T : blockIdx.x;
    if (T == 64 && waves == 1) id = blockIdx.x * (MOST / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const bool pre = !BRANCH || a.pre.kind, post = SUMS && a.post.kind, shared = BRANCH && !GROUPS && a.gate;
    float gain[N], times[N];
    Mask mask[V];
#pragma unroll
    for (int v = 0; v < V; v++) {
        team.parameters(a.pre.gain, v, 1.0f, gain + v * E);
        if constexpr (BRANCH) {
            float g[E];
            team.parameters(post ? a.post.gain : nullptr, v, 1.0f, times + v * E);
            team.parameters(shared ? (const float *)a.gate : nullptr, v, 1.0f, g);
#pragma unroll
            for (int i = 0; i < E; i++) times[v * E + i] *= g[i];
            if (a.drop.threshold) mask[v].init(a.drop, step_of(a.drop), team.counter(v));
        }
    }
    float acc[SUMS ? 4 : 2][N] = {};
    // GROUPS: the group's gate, and the group's sums of w fhat and w
    float q[GROUPS ? N : 1], by_f[GROUPS ? N : 1], plain[GROUPS ? N : 1];
    uint32_t group = ~0u;
    const float factor = a.beta * (a.drop.threshold ? a.drop.factor : 1.0f);

    Raw<TS> dsum[V], x[V], next_dsum[V] = {}, next_x[V] = {};
    Raw<TB> dout[V], f[V], next_dout[V] = {}, next_f[V] = {};
    float2 st = make_float2(0.0f, 1.0f), st_f = st, next_st = st, next_st_f = st;
    const auto fetch = [&](uint32_t r) {
#pragma unroll
        for (int v = 0; v < V; v++) {
            // zeros into registers of their own: what is on its way need not arrive first
            next_x[v] = next_dsum[v] = {};
            next_dout[v] = next_f[v] = {};
            team.pieces(v, [&](int p) {
                if (pre) {
                    team.template load<STREAM>(next_x[v], (const TS *)a.sum + r * a.ld_sum, v, p);
                    team.template load<STREAM>(next_dout[v], (const TB *)a.dout + r * a.ld_dout, v, p);
                }
                if (a.dsum) team.template load<STREAM>(next_dsum[v], (const TS *)a.dsum + r * a.ld_dsum, v, p);
                if (SUMS && a.f) team.template load<STREAM>(next_f[v], (const TB *)a.f + r * a.ld_f, v, p);
            });
        }
        if (pre) next_st = a.stats[r];
        if (post) next_st_f = a.stats[a.rows + r];
    };
    // rows id, id + all, ..; where groups of rows are summed, the `turns` ones from id * turns on
    const uint64_t first = GROUPS ? (uint64_t)id * a.turns : id;
    const uint32_t end = GROUPS ? (uint32_t)min(first + a.turns, (uint64_t)a.rows) : a.rows;
    uint32_t row = (uint32_t)min(first, (uint64_t)a.rows), begun = row;
    // two vectors of 16 waves leave no registers for a row on its way
    constexpr bool AHEAD = V == 1 || MOST == 256;
    // as in the forward pass: before the last stores of a row the next one's loads have arrived
    const auto arrived = [&] {
        if (!AHEAD) return;
#pragma unroll
        for (int v = 0; v < V; v++) {
            arrive(next_x[v]);
            arrive(next_dout[v]);
            arrive(next_dsum[v]);
            if constexpr (SUMS) arrive(next_f[v]);
        }
        asm volatile("" : "+v"(next_st.x), "+v"(next_st.y), "+v"(next_st_f.x), "+v"(next_st_f.y));
    };
    if (AHEAD && row < end) fetch(row);
    arrived();
    while (row < end) {
        if (!AHEAD) fetch(row);
#pragma unroll
        for (int v = 0; v < V; v++) {
            x[v] = next_x[v];
            dout[v] = next_dout[v];
            dsum[v] = next_dsum[v];
            f[v] = next_f[v];
        }
        st = next_st;
        st_f = next_st_f;
        const uint32_t at = row;
        row += GROUPS ? 1 : all;
        if (AHEAD && row < end) fetch(row);
        if constexpr (GROUPS) {
            if (at / a.gate_rows != group) {
                group = at / a.gate_rows;
#pragma unroll
                for (int v = 0; v < V; v++) {
                    Raw<TB> r = {};
                    team.pieces(v, [&](int p) { team.template load<false>(r, (const TB *)a.gate + group * a.ld_gate, v, p); });
                    team.unpack(r, v, q + v * E);
                    team.parameters(post ? a.post.gain : nullptr, v, 1.0f, times + v * E);
#pragma unroll
                    for (int i = v * E; i < (v + 1) * E; i++) {
                        times[i] *= q[i];
                        by_f[i] = plain[i] = 0.0f;
                    }
                }
            }
        }
        float d[N] = {};
        if (a.dsum)
#pragma unroll
            for (int v = 0; v < V; v++) team.unpack(dsum[v], v, d + v * E);
        if (pre) {
            float xhat[N], g[N], sg = 0.0f, sx = 0.0f;
#pragma unroll
            for (int v = 0; v < V; v++) {
                team.unpack(x[v], v, xhat + v * E);
                team.unpack(dout[v], v, g + v * E);
                // columns behind the row's end hold no gradient: whatever they add is zero
#pragma unroll
                for (int i = v * E; i < (v + 1) * E; i++) {
                    xhat[i] = (xhat[i] - team.about(v, i - v * E, st.x)) * st.y;
                    acc[0][i] = fmaf(g[i], xhat[i], acc[0][i]);
                    acc[1][i] += g[i];
                    g[i] *= gain[i];
                    sg += g[i];
                    sx = fmaf(g[i], xhat[i], sx);
                }
            }
            team.sum2(sg, sx);
            const float k0 = a.pre.kind == kNormLayer ? -sg * team.inv_width * st.y : 0.0f, k1 = -sx * team.inv_width * st.y;
#pragma unroll
            for (int i = 0; i < N; i++) d[i] += fmaf(g[i], st.y, fmaf(xhat[i], k1, k0));
        }
        if (!BRANCH) arrived();
#pragma unroll
        for (int v = 0; v < V; v++) {
            float o[E];
#pragma unroll
            for (int i = 0; i < E; i++) o[i] = a.alpha * d[v * E + i];
            team.pieces(v, [&](int p) { team.template store<true>((TS *)a.dh + at * a.ld_dh, v, p, o); });
        }
        if constexpr (BRANCH) {
            float fhat[N], sg = 0.0f, sx = 0.0f;
#pragma unroll
            for (int v = 0; v < V; v++) {
                float *w = d + v * E, *y = fhat + v * E;
                if (a.drop.threshold) {
                    mask[v].template apply<SPLIT>(a.drop, at, factor, w);
                } else {
#pragma unroll
                    for (int i = 0; i < E; i++) w[i] *= factor;
                }
                if constexpr (SUMS) {
                    team.unpack(f[v], v, y);
#pragma unroll
                    for (int i = 0; i < E; i++) y[i] = (y[i] - team.about(v, i, st_f.x)) * st_f.y;
                }
                if constexpr (SUMS)
#pragma unroll
                    for (int i = 0; i < E; i++) {
                        float &s = GROUPS ? by_f[GROUPS ? v * E + i : 0] : acc[2][v * E + i],
                              &t = GROUPS ? plain[GROUPS ? v * E + i : 0] : acc[3][v * E + i];
                        s = fmaf(w[i], y[i], s);
                        t += w[i];
                    }
#pragma unroll
                for (int i = 0; i < E; i++) {
                    w[i] *= times[v * E + i];
                    if constexpr (SUMS) {
                        sg += w[i];
                        sx = fmaf(w[i], y[i], sx);
                    }
                }
            }
            if (post) {
                team.sum2(sg, sx);
                const float k0 = a.post.kind == kNormLayer ? -sg * team.inv_width * st_f.y : 0.0f, k1 = -sx * team.inv_width * st_f.y;
#pragma unroll
                for (int i = 0; i < N; i++) d[i] = fmaf(d[i], st_f.y, fmaf(fhat[i], k1, k0));
            }
            arrived();
#pragma unroll
            for (int v = 0; v < V; v++) team.pieces(v, [&](int p) { team.template store<true>((TB *)a.df + at * a.ld_df, v, p, d + v * E); });
        }
        if constexpr (GROUPS) {
            const uint32_t start = group * a.gate_rows;
            const bool ends = at + 1 == a.rows || at + 1 - start == a.gate_rows;
            if (ends || at + 1 == end) {
#pragma unroll
                for (int i = 0; i < N; i++) {
                    acc[2][i] = fmaf(q[i], by_f[i], acc[2][i]);
                    acc[3][i] = fmaf(q[i], plain[i], acc[3][i]);
                }
                if (a.dgate) {
                    float *to = ends && begun == start ? a.dgate + group * a.ld_dgate : a.edge + ((uint64_t)(begun == start) * all + id) * a.width;
#pragma unroll
                    for (int v = 0; v < V; v++) {
                        float g[E], b[E];
                        team.parameters(post ? a.post.gain : nullptr, v, 1.0f, g);
                        team.parameters(post ? a.post.bias : nullptr, v, 0.0f, b);
#pragma unroll
                        for (int i = 0; i < E; i++) g[i] = fmaf(g[i], by_f[v * E + i], b[i] * plain[v * E + i]);
                        team.pieces(v, [&](int p) { team.template store<false>(to, v, p, g); });
                    }
                }
                begun = at + 1;
            }
        }
    }
    // The workgroup's part of each sum: its teams' in a fixed order.
    uint32_t sum = 0, wanted = __popc(a.want);
#pragma unroll
    for (int s = 0; s < (SUMS ? 4 : 2); s++) {
        if (!(a.want >> s & 1)) continue;
        float *to = a.part + ((uint64_t)blockIdx.x * wanted + sum++) * a.width;
        if (T == 64 && waves > 1) {
#pragma unroll
            for (int v = 0; v < V; v++) team.pieces(v, [&](int p) { team.template store<false>(to, v, p, acc[s] + v * E); });
        } else {  // four waves of whole teams
#pragma unroll
            for (int off = T; off < 64; off <<= 1)
#pragma unroll
                for (int i = 0; i < N; i++) acc[s][i] += __shfl_xor(acc[s][i], off, 64);
            __syncthreads();
            if ((threadIdx.x & 63) < T)
#pragma unroll
                for (int v = 0; v < V; v++)
#pragma unroll
                    for (int i = 0; i < E; i++)
                        cells[threadIdx.x / 64 * T * N + (SPLIT ? team.column(v, i / 4) + i % 4 : team.column(v) + i)] = acc[s][v * E + i];
            __syncthreads();
            for (uint32_t c = threadIdx.x; c < a.width; c += 256)
                to[c] = (cells[c] + cells[T * N + c]) + (cells[2 * T * N + c] + cells[3 * T * N + c]);
        }
    }
}

template <typename TS, typename TB>
void launch_grad(const ResidualGradArgs &a, hipStream_t s) {
    const int mode = grad_mode(a);
    const RowShape r = grad_shape(a.width, mode, a.f32);
    const size_t streams = (a.dsum ? sizeof(TS) : 0) + (a.pre.kind ? sizeof(TS) + sizeof(TB) : 0) + (a.f ? sizeof(TB) : 0);
    const bool stream = (uint64_t)a.rows * a.width * streams >= kStreamBytes;
    with_shape(r, [&](auto sh) {
        with_mode(mode, [&](auto m) {
            typedef decltype(sh) S;
            constexpr int MODE = decltype(m)::value;
            if constexpr (S::V == 1 || S::MOST == 1024 || MODE < (sizeof(TS) == 4 ? 2 : 3))  // what grad_shape gives
                with_access<S>(ragged_row(a.width, sizeof(TS) == 4), stream, [&](auto streaming, auto ragged) {
                    residual_grad_kernel<TS, TB, S::T, S::V, S::MOST, MODE, decltype(streaming)::value, decltype(ragged)::value>
                        <<<a.groups, r.threads, 0, s>>>(a, r.waves(), a.groups * r.teams());
                });
        });
    });
}

}  // namespace dedloc
