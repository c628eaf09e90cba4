// gfx950 kernels of dropout, and what joins the parts of the gradients of norms
// and of the ends of a block; those themselves are in block_forward.h and block_grad.h.
#include <algorithm>

#include "block_rows.h"

namespace dedloc {

// ------------------------------------------------------------------- dropout

// A thread keeps its columns (eight; four of fp32, so that every access of a wave is one piece of memory) and goes down the rows:
// `down` rows of `across` threads at a time (or, where a row has more than kDropThreads, a workgroup for
// each kDropThreads of them), kDropBatch rows loaded before the first is written.  Two threads of four columns share a
// counter: the even one draws the first of two rows, the odd one the second.  Bound by memory: 131072 x 512 bf16 44 us, 6.1 TB/s
// (p = 0, a plain copy, 2 GiB: 5.9); 65536 x 2048 fp32 174 us, 6.2 TB/s; 131072 x 333 fp16 33 us, 5.3 TB/s.  The
// generator's products were the bound before a thread kept its columns (20 of them a counter, 15 now).
template <typename T, bool STREAM, bool RAGGED>
__global__ __launch_bounds__(kDropThreads) void dropout_kernel(DropoutArgs a) {
    constexpr bool SPLIT = sizeof(T) == 4;
    constexpr int P = SPLIT ? 4 : E;
    const uint32_t row_in = threadIdx.x / a.across, place = blockIdx.y * kDropThreads + threadIdx.x - row_in * a.across;
    const uint32_t c = place * P;
    if (row_in >= a.down || c >= (a.width + E - 1) / E * E) return;  // pairs of threads stay together
    const uint64_t begin = (uint64_t)blockIdx.x * a.per, end = min(begin + a.per, (uint64_t)a.rows);
    const T *x = (const T *)a.x;
    T *out = (T *)a.out;
    Mask mask;
    if (a.drop.threshold) mask.init(a.drop, step_of(a.drop), place * P / E);
    for (uint64_t row = begin + row_in; row < end; row += (uint64_t)kDropBatch * a.down) {
        T r[kDropBatch][P];
#pragma unroll
        for (uint32_t k = 0; k < kDropBatch; k++) {
            const uint64_t at = min(row + k * a.down, end - 1);
            load_part<P, STREAM, RAGGED>(x + at * a.ld_x, c, a.width, r[k]);
        }
#pragma unroll
        for (uint32_t k = 0; k < kDropBatch; k += SPLIT ? 2 : 1) {
            float v[E];
#pragma unroll
            for (int i = 0; i < E; i++) v[i] = (float)r[k + i / P][i % P];
            if constexpr (RAGGED)
#pragma unroll
                for (int i = 0; i < E; i += P) align<P>(v + i, c, a.width);
            const uint64_t at = row + k * a.down;
            if (at >= end) break;
            if (a.drop.threshold) {
                const bool second = SPLIT && (threadIdx.x & 1);
                mask.template apply<SPLIT>(a.drop, (uint32_t)at + (second ? a.down : 0), a.drop.factor, v);
            }
            store_part<P, true, RAGGED>(out + at * a.ld_out, c, a.width, v);
            if (SPLIT && at + a.down < end) store_part<P, true, RAGGED>(out + (at + a.down) * a.ld_out, c, a.width, v + 4);
        }
    }
}

hipError_t launch_dropout(int dtype, DropoutArgs a, hipStream_t s) {
    const uint32_t vectors = (a.width + E - 1) / E * (dtype == kF32 ? 2 : 1);  // threads of a row
    uint32_t threads = kDropThreads, pieces = 1;
    a.across = vectors;
    a.down = 1;
    if (vectors > kDropThreads) {
        a.across = kDropThreads;
        pieces = (vectors + kDropThreads - 1) / kDropThreads;
    } else {  // the workgroup with the fewest idle threads
        uint32_t best = 0;
        for (uint32_t n = 256; n <= kDropThreads; n += 64)
            if (n >= vectors && n / vectors * vectors * 1024 / n > best) {
                best = n / vectors * vectors * 1024 / n;
                threads = n;
            }
        a.down = threads / vectors;
    }
    // rows of a workgroup: whole batches where the rows are many, else as many workgroups as fill the GPU
    const uint64_t turns = (a.rows + a.down - 1) / a.down;
    const uint32_t deep = (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(kDropBatch, turns * pieces / kDropGroups));
    a.per = (uint32_t)std::max<uint64_t>((uint64_t)deep * a.down, (a.rows + kBlockGrid - 1) / kBlockGrid);
    const dim3 groups((a.rows + a.per - 1) / a.per, pieces);
    const auto go = [&](auto t) {
        typedef decltype(t) T;
        with_access<Shape<64, 1, 256>>(a.width % E, (uint64_t)a.rows * a.width * sizeof(T) >= kStreamBytes, [&](auto streaming, auto ragged) {
            dropout_kernel<T, decltype(streaming)::value, decltype(ragged)::value><<<groups, threads, 0, s>>>(a);
        });
    };
    if (dtype == kF32)
        go(0.0f);
    else if (dtype == kFP16)
        go(_Float16());
    else
        go(__bf16());
    return hipGetLastError();
}

// ------------------------------------------------------------- joins of parts

// The parts of all workgroups, joined in 64 bits: 16 columns of a sum to a workgroup, four a thread, 256 parts at a time.  The learned
// gate's gradient is gain * (sum of w fhat) + bias * (sum of w); where it takes both sums one workgroup has them.  4 us for
// the parts of 8192 x 1024, 15 for those of four sums of 65536 x 2048 (34 MB); 32 columns and two sums a workgroup took 17 for the first.
__global__ __launch_bounds__(1024) void residual_join_kernel(ResidualGradArgs a) {
    __shared__ double cells[256][17];
    const uint32_t x = threadIdx.x & 3, y = threadIdx.x >> 2, c = blockIdx.x * 16 + x * 4, wanted = __popc(a.want);
    const bool shared = a.gate && !a.gate_rows, both = shared && a.dgate && a.post.bias;
    uint32_t first = 0;  // the blockIdx.y'th wanted sum
    for (uint32_t left = blockIdx.y; left || !(a.want >> first & 1); first++) left -= a.want >> first & 1;
    if (first == 3 && both && (a.want & 4)) return;
    double total[2] = {};
    for (uint32_t s = first; s < (first == 2 && both ? 4 : first + 1); s++) {
        const float *from = a.part + (uint64_t)__popc(a.want & ((1u << s) - 1)) * a.width + c;
        double t[4] = {};
        if (c + 4 <= a.width) {
#pragma unroll 4
            for (uint32_t p = y; p < a.groups; p += 256) {
                float v[4];
                load_part<4, false, false>(from + (uint64_t)p * wanted * a.width, 0, 4, v);
#pragma unroll
                for (int i = 0; i < 4; i++) t[i] += (double)v[i];
            }
        } else {
            for (uint32_t p = y; p < a.groups; p += 256)
#pragma unroll
                for (uint32_t i = 0; i < 4; i++)
                    if (c + i < a.width) t[i] += (double)from[(uint64_t)p * wanted * a.width + i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; i++) cells[y][x * 4 + i] = t[i];
        __syncthreads();
        // 64 threads to a step of 16 columns: four parts each, then four each of those, then the last 16
        const uint32_t col = threadIdx.x & 15, part = threadIdx.x >> 4;
        double u = (cells[part * 4][col] + cells[part * 4 + 1][col]) + (cells[part * 4 + 2][col] + cells[part * 4 + 3][col]);
        __syncthreads();
        cells[part][col] = u;
        __syncthreads();
        if (part < 16) {
            u = (cells[part * 4][col] + cells[part * 4 + 1][col]) + (cells[part * 4 + 2][col] + cells[part * 4 + 3][col]);
            cells[64 + part][col] = u;
        }
        __syncthreads();
        if (part == 0) {
            u = 0.0;
            for (int p = 0; p < 16; p++) u += cells[64 + p][col];
            total[s - first] = u;
        }
    }
    const uint32_t at = blockIdx.x * 16 + threadIdx.x;
    if (threadIdx.x >= 16 || at >= a.width) return;
    const auto add = [&](float *to, double v) {
        if (to) to[at] = fmaf(a.samples, (float)v, to[at]);
    };
    if (first == 0) add(a.dpre_gain, total[0]);
    if (first == 1) add(a.dpre_bias, total[0]);
    const double gate = shared ? (double)((const float *)a.gate)[at] : 1.0;
    if (first == 2) {
        add(a.dpost_gain, gate * total[0]);
        if (both) add(a.dpost_bias, gate * total[1]);
        if (shared) add(a.dgate, (a.post.gain ? (double)a.post.gain[at] : 1.0) * total[0] + (both ? (double)a.post.bias[at] * total[1] : 0.0));
    }
    if (first == 3) add(a.dpost_bias, gate * total[0]);
}

// The gate's gradient of groups of rows that more than one team has: team `id` holds the start, the next ones the rest.
// A workgroup per group, or, where teams are fewer, per team: of those that start in its range only the last can be cut.
__global__ __launch_bounds__(1024) void gate_join_kernel(ResidualGradArgs a, uint32_t all, bool by_group) {
    __shared__ float cells[16][64];
    const uint32_t x = threadIdx.x & 63, y = threadIdx.x >> 6, c = blockIdx.y * 64 + x;
    uint32_t group = blockIdx.x;
    if (!by_group) {
        const uint64_t begin = (uint64_t)blockIdx.x * a.turns, end = min(begin + a.turns, (uint64_t)a.rows);
        if (begin >= end) return;
        group = (uint32_t)((end - 1) / a.gate_rows);
        if ((uint64_t)group * a.gate_rows < begin) return;  // another team's
    }
    const uint64_t from = (uint64_t)group * a.gate_rows, to = min(from + a.gate_rows, (uint64_t)a.rows);
    const uint32_t id = (uint32_t)(from / a.turns), last = (uint32_t)((to - 1) / a.turns);
    if (id == last) return;  // whole
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

// fp32 streams go with any branch, 16-bit ones with a branch of their type.
template <typename F>
static void with_types(int stream, int branch, F f) {
    if (stream == kF32) {
        if (branch == kF32) return f(0.0f, 0.0f);
        if (branch == kFP16) return f(0.0f, _Float16());
        return f(0.0f, __bf16());
    }
    if (stream == kFP16) return f(_Float16(), _Float16());
    f(__bf16(), __bf16());
}

hipError_t launch_residual(int stream, int branch, const ResidualArgs &a, hipStream_t s) {
    with_types(stream, branch, [&](auto ts, auto tb) { launch_forward<decltype(ts), decltype(tb)>(a, s); });
    return hipGetLastError();
}

hipError_t launch_residual_grad(int stream, int branch, const ResidualGradArgs &a, hipStream_t s) {
    with_types(stream, branch, [&](auto ts, auto tb) { launch_grad<decltype(ts), decltype(tb)>(a, s); });
    return hipGetLastError();
}

hipError_t launch_residual_join(const ResidualGradArgs &a, hipStream_t s) {
    residual_join_kernel<<<dim3((a.width + 15) / 16, __builtin_popcount(a.want)), 1024, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_gate_join(const ResidualGradArgs &a, hipStream_t s) {
    if (a.turns % a.gate_rows == 0) return hipSuccess;  // no range of rows cuts a group
    // gate_rows may be any number of 32 bits: no sum with it
    const uint32_t all = a.groups * grad_shape(a.width, 3, a.f32).teams(), gates = (a.rows - 1) / a.gate_rows + 1;
    gate_join_kernel<<<dim3(std::min(all, gates), (a.width + 63) / 64), 1024, 0, s>>>(a, all, gates < all);
    return hipGetLastError();
}

}  // namespace dedloc
