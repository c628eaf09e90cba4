// gfx950 kernels of what stands between the matrix products of a model's step:
// dropout, norms of rows, and the end of one block with the start of the next
// in one pass (the branch's norm, gate, dropout, the residual sum and its norm),
// with their gradients.  All of it is bound by the bytes of the rows: a row is
// read once, held in registers by the threads that share it, and written once.
#include <algorithm>

#include "block_internal.h"
#include "ops_internal.h"

namespace dedloc {

namespace {

constexpr int E = 8;  // columns of a vector: one counter of the generator, 16 bytes of a 16-bit type

// N elements at any alignment of the element, as floats and back.
template <int N, typename T>
struct Vec {
    T v[N];
} __attribute__((packed, aligned(sizeof(T))));

// Columns c to c + 7 of a row, zeros behind its end.
template <typename T>
__device__ inline void load(const T *row, uint32_t c, uint32_t width, float *o) {
    if (c + E <= width) {
        const Vec<E, T> q = *(const Vec<E, T> *)(row + c);
#pragma unroll
        for (int i = 0; i < E; i++) o[i] = (float)q.v[i];
    } else {
#pragma unroll
        for (int i = 0; i < E; i++) o[i] = c + i < width ? (float)row[c + i] : 0.0f;
    }
}
template <typename T>
__device__ inline void store(T *row, uint32_t c, uint32_t width, const float *o) {
    if (c + E <= width) {
        Vec<E, T> q;
#pragma unroll
        for (int i = 0; i < E; i++) q.v[i] = (T)o[i];
        *(Vec<E, T> *)(row + c) = q;
    } else {
#pragma unroll
        for (int i = 0; i < E; i++)
            if (c + i < width) row[c + i] = (T)o[i];
    }
}

// fp32 v rounded to T and back: the result of the fp32 operation before it (without this an fp16 one becomes a single
// instruction with a rounding of its own).
template <typename T>
__device__ inline float rounded(float v) {
    if constexpr (sizeof(T) == 2) asm("" : "+v"(v));
    return (float)(T)v;
}

// ------------------------------------------------------------------ the mask

// Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011): ten rounds of two
// 32 by 32 bit products.  A counter gives eight 16-bit numbers, one for each column of a vector, so the mask of a
// 16-bit type costs one counter for 16 bytes.
__device__ inline void philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1, uint32_t *o) {
#pragma unroll
    for (int r = 0; r < 10; r++) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    o[0] = c0;
    o[1] = c1;
    o[2] = c2;
    o[3] = c3;
}

__device__ inline uint32_t step_of(const DropArgs &d) { return d.step + (d.step_at ? (uint32_t)*d.step_at : 0u); }

// What is dropped is zero, whatever it held: an infinity or NaN does not pass.
__device__ inline void drop(const DropArgs &d, uint32_t step, uint32_t row, uint32_t c, float factor, float *x) {
    uint32_t w[4];
    philox(c / E, d.row0 + row, d.site, step, d.key0, d.key1, w);
#pragma unroll
    for (int i = 0; i < E; i++) {
        const uint32_t half = i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu;
        x[i] = half < d.threshold ? 0.0f : x[i] * factor;
    }
}

// --------------------------------------------------------------- sums of a row

template <int CTRL>
__device__ inline float moved(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}

// The sum over aligned groups of T lanes, in all of them.
template <int T>
__device__ inline float lanes_sum(float v) {
    v += moved<0xB1>(v);                  // the other of a pair
    v += moved<0x4E>(v);                  // the other pair of four
    v += moved<0x141>(v);                 // eight, mirrored
    if (T >= 16) v += moved<0x140>(v);    // sixteen, mirrored
    if (T >= 32) {
        const auto p = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
        const unsigned x = p[0], y = p[1];  // a bit cast of an element itself takes the first
        v = __builtin_bit_cast(float, x) + __builtin_bit_cast(float, y);
    }
    if (T >= 64) {
        const auto p = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
        const unsigned x = p[0], y = p[1];
        v = __builtin_bit_cast(float, x) + __builtin_bit_cast(float, y);
    }
    return v;
}
template <int T>
__device__ inline double lanes_sum(double v) {
#pragma unroll
    for (int off = 1; off < T; off <<= 1) v += __shfl_xor(v, off, 64);
    return v;
}

// The threads that share a row: T lanes of a wave (T < 64), or `waves` whole waves, then the workgroup
// where there is more than one.  Waves meet in two sets of words in turn: a set is written again only after the barrier
// of the other, which every wave reaches after its reads of the first.
constexpr int kMaxWaves = 16;
struct Meet {
    double a[2][kMaxWaves], b[2][kMaxWaves];
};

template <int T, int V>
struct Team {
    uint32_t t, lanes, waves, wave, width;
    Meet *meet;
    mutable int turn;

    __device__ Team(uint32_t row_waves, uint32_t width_, Meet *m) : waves(T < 64 ? 1 : row_waves), width(width_), meet(m), turn(0) {
        lanes = T * waves;
        t = threadIdx.x & (lanes - 1);
        wave = waves > 1 ? threadIdx.x / 64 : 0;
    }
    __device__ uint32_t column(int v) const { return (v * lanes + t) * E; }
    // columns of a row that wave w of it holds
    __device__ uint32_t held(uint32_t w) const {
        uint32_t n = 0;
#pragma unroll
        for (int v = 0; v < V; v++) {
            const uint32_t c = (v * lanes + w * T) * E;
            n += c >= width ? 0 : min(width - c, (uint32_t)(T * E));
        }
        return n;
    }
    template <typename F>
    __device__ void sum2(F &a, F &b) const {
        a = lanes_sum<T>(a);
        b = lanes_sum<T>(b);
        if (waves == 1) return;
        F *pa = (F *)meet->a[turn], *pb = (F *)meet->b[turn];
        if ((threadIdx.x & 63) == 0) {
            pa[wave] = a;
            pb[wave] = b;
        }
        __syncthreads();
        a = b = 0;
        for (uint32_t w = 0; w < waves; w++) {
            a += pa[w];
            b += pb[w];
        }
        turn ^= 1;
    }
    // (sum of x, sum of squares about the mean) from the waves' own: no subtraction of large squares.
    __device__ void moments(const float *x, float &mean, float &m2) const {
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < V * E; i++) s += x[i];
        s = lanes_sum<T>(s);
        const uint32_t n = held(wave);
        const float own = n ? s / (float)n : 0.0f;
        float q = lanes_sum<T>(squares(x, own));
        mean = own;
        m2 = q;
        if (waves == 1) return;
        float *pa = (float *)meet->a[turn], *pb = (float *)meet->b[turn];
        if ((threadIdx.x & 63) == 0) {
            pa[wave] = s;
            pb[wave] = q;
        }
        __syncthreads();
        s = 0.0f;
        for (uint32_t w = 0; w < waves; w++) s += pa[w];
        mean = s / (float)width;
        m2 = 0.0f;
        for (uint32_t w = 0; w < waves; w++) {
            const uint32_t k = held(w);
            const float d = k ? pa[w] / (float)k - mean : 0.0f;
            m2 += pb[w] + (float)k * d * d;
        }
        turn ^= 1;
    }
    template <typename F>
    __device__ F squares(const float *x, F about) const {
        F q = 0;
#pragma unroll
        for (int v = 0; v < V; v++) {
            const uint32_t c = column(v);
#pragma unroll
            for (int i = 0; i < E; i++) {
                const F d = (F)x[v * E + i] - about;
                if (c + i < width) q = fma(d, d, q);
            }
        }
        return q;
    }
    // The statistics of a norm.  Sums of squares that leave fp32 (entries above 1e18) are taken again in 64 bits;
    // every thread of the row sees the same sum, so all take that way or none.
    __device__ float2 stats(const float *x, const NormArgs &n) const {
        float mean = 0.0f, m2 = 0.0f;
        if (n.kind == kNormLayer) {
            moments(x, mean, m2);
        } else {
            float none = 0.0f;
            m2 = squares(x, 0.0f);
            sum2(m2, none);
        }
        float var = m2 / (float)width;
        if (!(m2 < 0x1p120f)) {
            double s = 0.0, none = 0.0;
            if (n.kind == kNormLayer) {
#pragma unroll
                for (int i = 0; i < V * E; i++) s += (double)x[i];
                sum2(s, none);
                s /= (double)width;
                mean = (float)s;
            }
            double q = squares(x, s);
            none = 0.0;
            sum2(q, none);
            return make_float2(mean, (float)(1.0 / sqrt(q / (double)width + (double)n.eps)));
        }
        return make_float2(mean, 1.0f / sqrtf(var + n.eps));
    }
};

// A vector of parameters at columns c to c + 7; `other` where there is none.
__device__ inline void parameters(const float *p, uint32_t c, uint32_t width, float other, float *o) {
    if (p) {
        load<float>(p, c, width, o);
    } else {
#pragma unroll
        for (int i = 0; i < E; i++) o[i] = other;
    }
}
template <typename TB>
__device__ inline void gates(const void *gate, uint64_t ld, uint32_t gate_rows, uint32_t row, uint32_t c, uint32_t width, float *o) {
    if (gate_rows)
        load<TB>((const TB *)gate + (uint64_t)(row / gate_rows) * ld, c, width, o);
    else
        load<float>((const float *)gate, c, width, o);
}

}  // namespace

// ------------------------------------------------------------------- dropout

// A workgroup takes `per` rows at a time, a thread every 256th vector of them; rows of more than kDropVectors vectors go
// to several workgroups.
template <typename T>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs a) {
    const uint32_t vectors = (a.width + E - 1) / E, step = step_of(a.drop);
    for (uint64_t row0 = (uint64_t)blockIdx.x * a.per; row0 < a.rows; row0 += (uint64_t)gridDim.x * a.per) {
        const uint32_t rows = min(a.per, a.rows - (uint32_t)row0), begin = blockIdx.y * kDropVectors;
        const uint32_t end = min(rows * vectors, begin + kDropVectors);
        for (uint32_t i = begin + threadIdx.x; i < end; i += 256) {
            const uint32_t r = a.per == 1 ? 0 : vectors == 1 ? i : (uint32_t)(((uint64_t)i * a.magic) >> 32);
            const uint32_t c = (i - r * vectors) * E, row = (uint32_t)row0 + r;
            float v[E];
            load<T>((const T *)a.x + row * a.ld_x, c, a.width, v);
            if (a.drop.threshold) drop(a.drop, step, row, c, a.drop.factor, v);
            store<T>((T *)a.out + row * a.ld_out, c, a.width, v);
        }
    }
}

// -------------------------------------------------------- forward: norm, residual

template <typename TS, typename TB, int T, int V, int MOST>
__global__ __launch_bounds__(MOST) void residual_kernel(ResidualArgs a, uint32_t waves) {
    __shared__ Meet meet;
    const Team<T, V> team(waves, a.width, &meet);
    const uint32_t teams = blockDim.x / team.lanes, step = step_of(a.drop);
    for (uint64_t row0 = (uint64_t)blockIdx.x * teams; row0 < a.rows; row0 += (uint64_t)gridDim.x * teams) {
        const uint32_t row = (uint32_t)row0 + threadIdx.x / team.lanes;
        const bool live = row < a.rows;  // the others go along: sums are taken over whole waves
        const uint64_t at = live ? row : a.rows - 1;
        float x[V * E];
#pragma unroll
        for (int v = 0; v < V; v++) load<TS>((const TS *)a.h + at * a.ld_h, team.column(v), a.width, x + v * E);
        if (a.f) {
            float f[V * E];
#pragma unroll
            for (int v = 0; v < V; v++) load<TB>((const TB *)a.f + at * a.ld_f, team.column(v), a.width, f + v * E);
            if (a.post.kind) {
                const float2 st = team.stats(f, a.post);
                if (a.stats && live && team.t == 0) a.stats[a.rows + row] = st;
#pragma unroll
                for (int v = 0; v < V; v++) {
                    float g[E], b[E];
                    parameters(a.post.gain, team.column(v), a.width, 1.0f, g);
                    parameters(a.post.bias, team.column(v), a.width, 0.0f, b);
#pragma unroll
                    for (int i = 0; i < E; i++) f[v * E + i] = fmaf((f[v * E + i] - st.x) * st.y, g[i], b[i]);
                }
            }
#pragma unroll
            for (int v = 0; v < V; v++) {
                if (a.gate) {
                    float g[E];
                    gates<TB>(a.gate, a.ld_gate, a.gate_rows, (uint32_t)at, team.column(v), a.width, g);
#pragma unroll
                    for (int i = 0; i < E; i++) f[v * E + i] *= g[i];
                }
                if (a.drop.threshold) drop(a.drop, step, (uint32_t)at, team.column(v), a.drop.factor, f + v * E);
#pragma unroll
                for (int i = 0; i < E; i++) x[v * E + i] = fmaf(a.beta, f[v * E + i], a.alpha * x[v * E + i]);
            }
            // the norm sees the sum as it is stored
#pragma unroll
            for (int i = 0; i < V * E; i++) x[i] = rounded<TS>(x[i]);
            if (a.sum && live)
#pragma unroll
                for (int v = 0; v < V; v++) store<TS>((TS *)a.sum + at * a.ld_sum, team.column(v), a.width, x + v * E);
        }
        if (!a.pre.kind) continue;
        const float2 st = team.stats(x, a.pre);
        if (!live) continue;
        if (a.stats && team.t == 0) a.stats[row] = st;
#pragma unroll
        for (int v = 0; v < V; v++) {
            float g[E], b[E];
            parameters(a.pre.gain, team.column(v), a.width, 1.0f, g);
            parameters(a.pre.bias, team.column(v), a.width, 0.0f, b);
#pragma unroll
            for (int i = 0; i < E; i++) x[v * E + i] = fmaf((x[v * E + i] - st.x) * st.y, g[i], b[i]);
            store<TB>((TB *)a.out + at * a.ld_out, team.column(v), a.width, x + v * E);
        }
    }
}

// ----------------------------------------------------------------- gradients

// d of a norm's input from g = gain * dy, xhat and the means of g and g * xhat.
template <int N>
__device__ inline void norm_back(const float *g, const float *xhat, float mean_g, float mean_gx, float rstd, float *d) {
#pragma unroll
    for (int i = 0; i < N; i++) d[i] = rstd * (g[i] - mean_g - xhat[i] * mean_gx);
}

template <typename TS, typename TB, int T, int V, int MOST, bool BRANCH>
__global__ __launch_bounds__(MOST) void residual_grad_kernel(ResidualGradArgs a, uint32_t waves) {
    constexpr int N = V * E;
    __shared__ Meet meet;
    __shared__ float cells[T < 64 ? 4 * T * E : MOST == 256 ? 4 * 64 * N : 1];
    const Team<T, V> team(waves, a.width, &meet);
    const uint32_t teams = blockDim.x / team.lanes, id = blockIdx.x * teams + threadIdx.x / team.lanes, all = a.groups * teams;
    const float inv = 1.0f / (float)a.width;
    const uint32_t step = BRANCH ? step_of(a.drop) : 0;
    float acc[BRANCH ? 4 : 2][N] = {}, gated[BRANCH ? N : 1] = {};
    const uint64_t first = a.cut ? (uint64_t)id * a.turns : id;
    const uint32_t stride = a.cut ? 1 : all;
    uint32_t begun = 0;  // cut: the first row of the current group, or of the range
    if (a.cut) begun = (uint32_t)min(first, (uint64_t)a.rows);
    for (uint32_t k = 0; k < a.turns; k++) {
        const uint64_t row = first + (uint64_t)k * stride;
        const bool live = row < a.rows;
        const uint64_t at = live ? row : a.rows - 1;
        float d[N] = {};
        if (a.dsum)
#pragma unroll
            for (int v = 0; v < V; v++) load<TS>((const TS *)a.dsum + at * a.ld_dsum, team.column(v), a.width, d + v * E);
        float f[N];
        if (BRANCH && a.f)
#pragma unroll
            for (int v = 0; v < V; v++) load<TB>((const TB *)a.f + at * a.ld_f, team.column(v), a.width, f + v * E);
        if (!BRANCH || a.pre.kind) {
            float x[N], g[N];
            const float2 st = a.stats[at];
#pragma unroll
            for (int v = 0; v < V; v++) {
                load<TS>((const TS *)a.sum + at * a.ld_sum, team.column(v), a.width, x + v * E);
                load<TB>((const TB *)a.dout + at * a.ld_dout, team.column(v), a.width, g + v * E);
            }
            float sg = 0.0f, sx = 0.0f;
#pragma unroll
            for (int v = 0; v < V; v++) {
                float gain[E];
                parameters(a.pre.gain, team.column(v), a.width, 1.0f, gain);
#pragma unroll
                for (int i = v * E; i < (v + 1) * E; i++) {
                    x[i] = (x[i] - st.x) * st.y;
                    if (live) {
                        acc[0][i] = fmaf(g[i], x[i], acc[0][i]);
                        acc[1][i] += g[i];
                    }
                    g[i] *= gain[i - v * E];
                    sg += g[i];
                    sx = fmaf(g[i], x[i], sx);
                }
            }
            team.sum2(sg, sx);
            sg = a.pre.kind == kNormLayer ? sg * inv : 0.0f;
            sx *= inv;
            float dx[N];
            norm_back<N>(g, x, sg, sx, st.y, dx);
#pragma unroll
            for (int i = 0; i < N; i++) d[i] += dx[i];
        }
        if (live)
#pragma unroll
            for (int v = 0; v < V; v++) {
                float o[E];
#pragma unroll
                for (int i = 0; i < E; i++) o[i] = a.alpha * d[v * E + i];
                store<TS>((TS *)a.dh + at * a.ld_dh, team.column(v), a.width, o);
            }
        if constexpr (BRANCH) {
            const float2 st = a.post.kind ? a.stats[a.rows + at] : make_float2(0.0f, 1.0f);
            float sg = 0.0f, sx = 0.0f;
#pragma unroll
            for (int v = 0; v < V; v++) {
                const uint32_t c = team.column(v);
                float gate[E], gain[E], bias[E];
#pragma unroll
                for (int i = v * E; i < (v + 1) * E; i++) d[i] *= a.beta;
                if (a.drop.threshold) drop(a.drop, step, (uint32_t)at, c, a.drop.factor, d + v * E);
                if (a.f)
#pragma unroll
                    for (int i = v * E; i < (v + 1) * E; i++) f[i] = (f[i] - st.x) * st.y;
                if (a.post.kind) parameters(a.post.gain, c, a.width, 1.0f, gain);
                if (a.gate) gates<TB>(a.gate, a.ld_gate, a.gate_rows, (uint32_t)at, c, a.width, gate);
                if (a.gate && a.gate_rows) {
                    if (a.dgate && live) {
                        if (a.post.kind) parameters(a.post.bias, c, a.width, 0.0f, bias);
#pragma unroll
                        for (int i = v * E; i < (v + 1) * E; i++) {
                            const float value = a.post.kind ? fmaf(f[i], gain[i - v * E], bias[i - v * E]) : f[i];
                            gated[i] = fmaf(d[i], value, gated[i]);
                        }
                    }
#pragma unroll
                    for (int i = v * E; i < (v + 1) * E; i++) d[i] *= gate[i - v * E];
                }
                if ((a.want & 12) && live)
#pragma unroll
                    for (int i = v * E; i < (v + 1) * E; i++) {
                        acc[2][i] = fmaf(d[i], f[i], acc[2][i]);
                        acc[3][i] += d[i];
                    }
                if (a.gate && !a.gate_rows)
#pragma unroll
                    for (int i = v * E; i < (v + 1) * E; i++) d[i] *= gate[i - v * E];
                if (a.post.kind)
#pragma unroll
                    for (int i = v * E; i < (v + 1) * E; i++) {
                        d[i] *= gain[i - v * E];
                        sg += d[i];
                        sx = fmaf(d[i], f[i], sx);
                    }
            }
            if (a.post.kind) {
                team.sum2(sg, sx);
                sg = a.post.kind == kNormLayer ? sg * inv : 0.0f;
                norm_back<N>(d, f, sg, sx * inv, st.y, d);
            }
            if (live)
#pragma unroll
                for (int v = 0; v < V; v++) store<TB>((TB *)a.df + at * a.ld_df, team.column(v), a.width, d + v * E);
            if (a.cut && a.dgate && live) {
                const uint32_t group = (uint32_t)at / a.gate_rows;
                const bool ends = at + 1 == a.rows || (at + 1) % a.gate_rows == 0;
                if (ends || k + 1 == a.turns) {
                    const bool whole = ends && begun == group * a.gate_rows;
                    float *to = whole ? a.dgate + group * a.ld_dgate
                                      : a.edge + ((uint64_t)(begun == group * a.gate_rows) * all + id) * a.width;
#pragma unroll
                    for (int v = 0; v < V; v++) store<float>(to, team.column(v), a.width, gated + v * E);
#pragma unroll
                    for (int i = 0; i < N; i++) gated[i] = 0.0f;
                    begun = (uint32_t)at + 1;
                }
            }
        }
    }
    // The workgroup's part of each sum: its teams' in a fixed order.
    uint32_t sum = 0, wanted = __popc(a.want);
#pragma unroll
    for (int s = 0; s < (BRANCH ? 4 : 2); s++) {
        if (!(a.want >> s & 1)) continue;
        float *to = a.part + ((uint64_t)blockIdx.x * wanted + sum++) * a.width;
        if (T == 64 && waves > 1) {
#pragma unroll
            for (int v = 0; v < V; v++) store<float>(to, team.column(v), a.width, acc[s] + v * E);
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
                    for (int i = 0; i < E; i++) cells[threadIdx.x / 64 * T * N + team.column(v) + i] = acc[s][v * E + i];
            __syncthreads();
            for (uint32_t c = threadIdx.x; c < a.width; c += 256)
                to[c] = (cells[c] + cells[T * N + c]) + (cells[2 * T * N + c] + cells[3 * T * N + c]);
        }
    }
}

// The parts of all workgroups in 64 bits, then the gradients: 16 columns to a workgroup, 64 parts at a time.
__global__ __launch_bounds__(1024) void residual_join_kernel(ResidualGradArgs a) {
    __shared__ double cells[64][17];
    const uint32_t x = threadIdx.x & 15, y = threadIdx.x >> 4, c = blockIdx.x * 16 + x, wanted = __popc(a.want);
    double total[kBlockSums] = {};
    uint32_t sum = 0;
#pragma unroll
    for (uint32_t s = 0; s < kBlockSums; s++) {
        if (!(a.want >> s & 1)) continue;
        double t = 0.0;
        if (c < a.width)
            for (uint32_t p = y; p < a.groups; p += 64) t += (double)a.part[((uint64_t)p * wanted + sum) * a.width + c];
        sum++;
        cells[y][x] = t;
        __syncthreads();
        for (uint32_t n = 32; n > 0; n >>= 1) {
            if (y < n) cells[y][x] += cells[y + n][x];
            __syncthreads();
        }
        total[s] = cells[0][x];
        __syncthreads();
    }
    if (y != 0 || c >= a.width) return;
    const auto add = [&](float *to, double v) {
        if (to) to[c] = fmaf(a.samples, (float)v, to[c]);
    };
    add(a.dpre_gain, total[0]);
    add(a.dpre_bias, total[1]);
    const bool shared = a.gate && !a.gate_rows;
    const double gate = shared ? (double)((const float *)a.gate)[c] : 1.0;
    add(a.dpost_gain, gate * total[2]);
    add(a.dpost_bias, gate * total[3]);
    if (shared && a.dgate) {
        const double gain = a.post.gain ? (double)a.post.gain[c] : 1.0, bias = a.post.bias ? (double)a.post.bias[c] : 0.0;
        add(a.dgate, gain * total[2] + bias * total[3]);
    }
}

// The gate's gradient of groups of rows that more than one team has: team `id` holds the start, the next ones the rest.
__global__ __launch_bounds__(1024) void gate_join_kernel(ResidualGradArgs a, uint32_t all) {
    __shared__ float cells[16][64];
    const uint32_t id = blockIdx.x, x = threadIdx.x & 63, y = threadIdx.x >> 6, c = blockIdx.y * 64 + x;
    const uint64_t begin = (uint64_t)id * a.turns, end = min(begin + a.turns, (uint64_t)a.rows);
    if (begin >= end) return;
    const uint32_t group = (uint32_t)((end - 1) / a.gate_rows);
    const uint64_t from = (uint64_t)group * a.gate_rows, to = min(from + a.gate_rows, (uint64_t)a.rows);
    if (from < begin || to <= end) return;  // another team's to join, or whole
    const uint32_t last = (uint32_t)((to - 1) / a.turns);
    float t = 0.0f;
    if (c < a.width)
        for (uint32_t k = id + y; k <= last; k += 16) t += a.edge[((uint64_t)(k == id) * all + k) * a.width + c];
    cells[y][x] = t;
    __syncthreads();
    for (uint32_t n = 8; n > 0; n >>= 1) {
        if (y < n) cells[y][x] += cells[y + n][x];
        __syncthreads();
    }
    if (y == 0 && c < a.width) a.dgate[group * a.ld_dgate + c] = cells[0][x];
}

// ------------------------------------------------------------------ launches

RowShape row_shape(uint32_t width) {
    if (width <= 64) return {8, 1, 256};
    if (width <= 128) return {16, 1, 256};
    if (width <= 256) return {32, 1, 256};
    uint32_t waves = 1;
    while (waves < 16 && waves * 512 < width) waves *= 2;
    return {64 * waves, waves * 512 < width ? 2u : 1u, waves == 1 ? 256 : 64 * waves};
}

hipError_t launch_dropout(int dtype, const DropoutArgs &a, hipStream_t s) {
    const dim3 groups(std::min((a.rows + a.per - 1) / a.per, kBlockGrid),
                      a.per == 1 ? ((a.width + E - 1) / E + kDropVectors - 1) / kDropVectors : 1);
    switch (dtype) {
        case kF32: dropout_kernel<float><<<groups, 256, 0, s>>>(a); break;
        case kFP16: dropout_kernel<_Float16><<<groups, 256, 0, s>>>(a); break;
        default: dropout_kernel<__bf16><<<groups, 256, 0, s>>>(a);
    }
    return hipGetLastError();
}

namespace {

// f(type of the stream, type of the branch): fp32 with any, a 16-bit type with itself.
template <typename F>
void with_types(int stream, int branch, F f) {
    if (stream == kF32) {
        if (branch == kF32) return f(0.0f, 0.0f);
        if (branch == kFP16) return f(0.0f, _Float16());
        return f(0.0f, __bf16());
    }
    if (stream == kFP16) return f(_Float16(), _Float16());
    f(__bf16(), __bf16());
}

template <int T_, int V_, int MOST_>
struct Shape {
    static constexpr int T = T_, V = V_, MOST = MOST_;
};
template <typename F>
void with_shape(const RowShape &r, F f) {
    if (r.lanes == 8) return f(Shape<8, 1, 256>());
    if (r.lanes == 16) return f(Shape<16, 1, 256>());
    if (r.lanes == 32) return f(Shape<32, 1, 256>());
    if (r.threads <= 256) return f(Shape<64, 1, 256>());
    if (r.vectors == 1) return f(Shape<64, 1, 1024>());
    f(Shape<64, 2, 1024>());
}

}  // namespace

hipError_t launch_residual(int stream, int branch, const ResidualArgs &a, hipStream_t s) {
    const RowShape r = row_shape(a.width);
    const uint32_t groups = std::min((a.rows + r.teams() - 1) / r.teams(), kBlockGrid), waves = r.lanes / 64;
    with_types(stream, branch, [&](auto ts, auto tb) {
        with_shape(r, [&](auto sh) {
            typedef decltype(sh) S;
            residual_kernel<decltype(ts), decltype(tb), S::T, S::V, S::MOST><<<groups, r.threads, 0, s>>>(a, waves);
        });
    });
    return hipGetLastError();
}

hipError_t launch_residual_grad(int stream, int branch, const ResidualGradArgs &a, hipStream_t s) {
    const RowShape r = row_shape(a.width);
    const uint32_t waves = r.lanes / 64;
    with_types(stream, branch, [&](auto ts, auto tb) {
        with_shape(r, [&](auto sh) {
            typedef decltype(sh) S;
            if (a.df)
                residual_grad_kernel<decltype(ts), decltype(tb), S::T, S::V, S::MOST, true><<<a.groups, r.threads, 0, s>>>(a, waves);
            else
                residual_grad_kernel<decltype(ts), decltype(tb), S::T, S::V, S::MOST, false><<<a.groups, r.threads, 0, s>>>(a, waves);
        });
    });
    return hipGetLastError();
}

hipError_t launch_residual_join(const ResidualGradArgs &a, hipStream_t s) {
    residual_join_kernel<<<(a.width + 15) / 16, 1024, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_gate_join(const ResidualGradArgs &a, hipStream_t s) {
    const uint32_t all = a.groups * row_shape(a.width).teams();
    gate_join_kernel<<<dim3(all, (a.width + 63) / 64), 1024, 0, s>>>(a, all);
    return hipGetLastError();
}

}  // namespace dedloc
