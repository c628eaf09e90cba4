// gfx950 kernels of the embedding lookup and its gradient.  Both move bytes:
// the lookup a row read and a row written per position, the gradient a row
// read per position and a row of the accumulator read and written per token.
//
// The gradient of a token is the sum of dy over its positions.  Positions are
// sorted by token (a stable radix sort, so equal tokens stay in ascending
// order), then summed in chunks of the sorted order: a run of equal tokens
// inside a chunk goes straight into the accumulator, one that a chunk's edge
// cuts leaves its parts in the workspace, joined in ascending order afterwards.
// No float atomics: the order of every sum, and so every bit, is fixed by the
// ids.  A token of half the positions costs as much time as many rare ones.
#include <algorithm>

#include "ops_internal.h"

namespace dedloc {

namespace {

__device__ inline float load1(const float *p) { return *p; }
__device__ inline float load1(const _Float16 *p) { return (float)*p; }
__device__ inline float load1(const __bf16 *p) { return (float)*p; }

// N elements at any alignment of the element, as floats and back.
template <int N, typename T>
struct Vec {
    T v[N];
} __attribute__((packed, aligned(sizeof(T))));

template <int N, typename T>
__device__ inline void load(const T *p, float *o) {
    const Vec<N, T> q = *(const Vec<N, T> *)p;
#pragma unroll
    for (int i = 0; i < N; i++) o[i] = (float)q.v[i];
}
template <int N, typename T>
__device__ inline void store(T *p, const float *o) {
    Vec<N, T> q;
#pragma unroll
    for (int i = 0; i < N; i++) q.v[i] = (T)o[i];
    *(Vec<N, T> *)p = q;
}

// The token at a position; `vocab` for an id outside the table.
__device__ inline uint32_t token(const void *ids, int wide, uint32_t vocab, uint32_t i) {
    const int64_t id = wide ? ((const int64_t *)ids)[i] : (int64_t)((const int32_t *)ids)[i];
    return id >= 0 && id < (int64_t)vocab ? (uint32_t)id : vocab;
}

}  // namespace

// A row of threads (tx of them, a power of two) per position, N elements per
// thread and turn.
template <typename TI, typename TO, int N>
__global__ __launch_bounds__(256) void embed_kernel(EmbedArgs a, uint32_t tx) {
    const uint32_t x = threadIdx.x & (tx - 1);
    const uint64_t row = (uint64_t)blockIdx.x * (256 / tx) + threadIdx.x / tx;
    if (row >= a.n) return;
    const uint32_t tok = token(a.ids, a.wide_ids, a.vocab, (uint32_t)row);
    const TI *from = (const TI *)a.table + (uint64_t)tok * a.ld_table;
    TO *to = (TO *)a.out + row * a.ld_out;
    const bool named = tok < a.vocab;
    for (uint32_t c = x * N; c < a.width; c += tx * N) {
        float v[N] = {};
        if (c + N <= a.width) {
            if (named) load<N>(from + c, v);
            for (int i = 0; i < N; i++) v[i] *= a.scale;
            if (!named) for (int i = 0; i < N; i++) v[i] = 0.0f;
            store<N>(to + c, v);
        } else {
            for (uint32_t i = c; i < a.width; i++) to[i] = (TO)(named ? load1(from + i) * a.scale : 0.0f);
        }
    }
}

// ------------------------------------------------------------------ the sort

// One pass orders the positions by 8 bits of their token, keeping the order of
// equal ones.  Chunk k counts its digits into counts[k][256].
template <bool FIRST>
__device__ inline uint2 pair_at(const EmbedGradArgs &a, const uint2 *from, uint32_t i) {
    if (FIRST) return make_uint2(token(a.ids, a.wide_ids, a.vocab, i), i);
    return from[i];
}

template <bool FIRST>
__global__ __launch_bounds__(256) void embed_count_kernel(EmbedGradArgs a, const uint2 *from, uint32_t shift) {
    __shared__ uint32_t count[256];
    count[threadIdx.x] = 0;
    __syncthreads();
    const uint32_t i0 = blockIdx.x * a.chunk, i1 = min(i0 + a.chunk, a.n);
    for (uint32_t i = i0 + threadIdx.x; i < i1; i += 256)
        atomicAdd(&count[(pair_at<FIRST>(a, from, i).x >> shift) & 255u], 1u);
    __syncthreads();
    a.counts[blockIdx.x * 256 + threadIdx.x] = count[threadIdx.x];
}

// Orders what one lane of a wave wrote to LDS before what another reads.
__device__ inline void wave_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

template <bool FIRST>
__global__ __launch_bounds__(256) void embed_scatter_kernel(EmbedGradArgs a, const uint2 *from, uint2 *to, uint32_t shift) {
    constexpr uint32_t R = kSortTile / 256;
    __shared__ uint32_t at[4][256];  // per wave and digit: where its next position goes
    __shared__ uint32_t total[4];
    const uint32_t t = threadIdx.x, lane = t & 63, wave = t >> 6, chunks = gridDim.x;
    // the first place of digit t: all smaller digits, and this digit in the chunks before
    uint32_t before = 0, all = 0;
    for (uint32_t k = 0; k < chunks; k++) {
        const uint32_t c = a.counts[k * 256 + t];
        all += c;
        before += k < blockIdx.x ? c : 0;
    }
    uint32_t scan = all;
    for (int off = 1; off < 64; off <<= 1) {
        const uint32_t up = __shfl_up(scan, off, 64);
        if (lane >= (uint32_t)off) scan += up;
    }
    if (lane == 63) total[wave] = scan;
    __syncthreads();
    uint32_t start = scan - all + before;
    for (uint32_t w = 0; w < wave; w++) start += total[w];
    const uint32_t end = min((blockIdx.x + 1) * a.chunk, a.n);
    for (uint32_t tile = blockIdx.x * a.chunk; tile < end; tile += kSortTile) {
        for (int w = 0; w < 4; w++) at[w][t] = 0;
        __syncthreads();
        // each wave takes a quarter of the tile, in order
        const uint32_t i0 = tile + wave * (kSortTile / 4) + lane;
        uint2 p[R];
#pragma unroll
        for (uint32_t r = 0; r < R; r++) {
            const uint32_t i = i0 + r * 64;
            p[r] = i < end ? pair_at<FIRST>(a, from, i) : make_uint2(0xffffffffu, 0u);
            if (i < end) atomicAdd(&at[wave][(p[r].x >> shift) & 255u], 1u);
        }
        __syncthreads();
        for (int w = 0; w < 4; w++) {
            const uint32_t c = at[w][t];
            at[w][t] = start;
            start += c;
        }
        __syncthreads();
#pragma unroll
        for (uint32_t r = 0; r < R; r++) {
            const bool in = i0 + r * 64 < end;
            const uint32_t digit = (p[r].x >> shift) & 255u;
            unsigned long long same = __ballot(in);
#pragma unroll
            for (int b = 0; b < 8; b++) {
                const unsigned long long m = __ballot((digit >> b) & 1u);
                same &= (digit >> b) & 1u ? m : ~m;
            }
            const uint32_t rank = __popcll(same & ((1ull << lane) - 1));
            if (in) to[at[wave][digit] + rank] = p[r];
            wave_order();
            if (in && rank == 0) at[wave][digit] += __popcll(same);
            wave_order();
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------ the sums

// A row of tx threads sums one chunk of kRunChunk sorted positions, four
// columns per thread.
template <typename T>
__global__ __launch_bounds__(256) void embed_sum_kernel(EmbedGradArgs a, const uint2 *pairs, uint32_t tx) {
    const uint32_t x = threadIdx.x & (tx - 1);
    const uint32_t chunk = blockIdx.x * (256 / tx) + threadIdx.x / tx;
    const uint64_t i0 = (uint64_t)chunk * kRunChunk;
    if (i0 >= a.n) return;
    const uint32_t i1 = (uint32_t)(i0 + kRunChunk < a.n ? i0 + kRunChunk : a.n);
    const uint32_t c = (blockIdx.y * tx + x) * 4;
    if (c >= a.width) return;
    const uint32_t live = min(4u, a.width - c);
    const T *dy = (const T *)a.dy + c;
    const uint32_t prev = i0 > 0 ? pairs[i0 - 1].x : 0xffffffffu, next = i1 < a.n ? pairs[i1].x : 0xffffffffu;
    float sum[4] = {};
    bool head = pairs[i0].x == prev;  // the run began in an earlier chunk
    for (uint32_t i = (uint32_t)i0; i < i1; i++) {
        const uint2 p = pairs[i];
        if (p.x == a.vocab) return;  // masked positions come last
        const T *row = dy + (uint64_t)p.y * a.ld_dy;
        float v[4] = {};
        if (live == 4) load<4>(row, v);
        else for (uint32_t e = 0; e < live; e++) v[e] = load1(row + e);
        for (int e = 0; e < 4; e++) sum[e] += v[e];
        const bool end = i + 1 == i1, more = (end ? next : pairs[i + 1].x) == p.x;
        if (more && !end) continue;
        float *to = head || more ? a.cut + ((uint64_t)chunk * 2 + (head ? 0 : 1)) * a.width + c
                                 : a.grad + (uint64_t)p.x * a.ld_grad + c;
        for (uint32_t e = 0; e < live; e++) to[e] = head || more ? sum[e] : fmaf(a.factor, sum[e], to[e]);
        head = false;
        for (int e = 0; e < 4; e++) sum[e] = 0.0f;
    }
}

// The run that leaves a chunk it began in: its parts, in ascending order.
__global__ __launch_bounds__(256) void embed_join_kernel(EmbedGradArgs a, const uint2 *pairs, uint32_t tx) {
    const uint32_t x = threadIdx.x & (tx - 1);
    uint64_t chunk = (uint64_t)blockIdx.x * (256 / tx) + threadIdx.x / tx;
    const uint64_t i1 = (chunk + 1) * kRunChunk;
    if (i1 >= a.n) return;
    const uint32_t tok = pairs[i1 - 1].x;
    if (tok == a.vocab || pairs[i1].x != tok) return;
    const uint64_t i0 = i1 - kRunChunk;
    if (i0 > 0 && pairs[i0].x == tok && pairs[i0 - 1].x == tok) return;  // it began earlier
    for (uint32_t c = x; c < a.width; c += tx) {
        float sum = a.cut[(chunk * 2 + 1) * a.width + c];
        for (uint64_t k = chunk + 1; k * kRunChunk < a.n && pairs[k * kRunChunk].x == tok; k++)
            sum += a.cut[k * 2 * a.width + c];
        float *to = a.grad + (uint64_t)tok * a.ld_grad + c;
        *to = fmaf(a.factor, sum, *to);
    }
}

// ---------------------------------------------------------------- launchers

namespace {

// Threads per row: the power of two that covers `units`, at most 256.
uint32_t row_threads(uint32_t units) {
    uint32_t tx = 1;
    while (tx < units && tx < 256) tx *= 2;
    return tx;
}

template <typename TI, typename TO>
void embed(const EmbedArgs &a, hipStream_t s) {
    constexpr int N = 16 / (sizeof(TI) > sizeof(TO) ? sizeof(TI) : sizeof(TO));
    const uint32_t tx = row_threads((a.width + N - 1) / N), rows = 256 / tx;
    embed_kernel<TI, TO, N><<<(a.n + rows - 1) / rows, 256, 0, s>>>(a, tx);
}
template <typename TI>
void embed(int out, const EmbedArgs &a, hipStream_t s) {
    if (out == kF32) embed<TI, float>(a, s);
    else if (out == kFP16) embed<TI, _Float16>(a, s);
    else embed<TI, __bf16>(a, s);
}

uint32_t sort_chunks(const EmbedGradArgs &a) { return (a.n + a.chunk - 1) / a.chunk; }
uint32_t run_chunks(const EmbedGradArgs &a) { return (a.n + kRunChunk - 1) / kRunChunk; }

}  // namespace

hipError_t launch_embed(int table, int out, const EmbedArgs &a, hipStream_t s) {
    if (table == kF32) embed<float>(out, a, s);
    else if (table == kFP16) embed<_Float16>(out, a, s);
    else embed<__bf16>(out, a, s);
    return hipGetLastError();
}

// from: the buffer that holds the pairs, or -1: the ids
hipError_t launch_embed_count(const EmbedGradArgs &a, int from, uint32_t shift, hipStream_t s) {
    if (from < 0) embed_count_kernel<true><<<sort_chunks(a), 256, 0, s>>>(a, nullptr, shift);
    else embed_count_kernel<false><<<sort_chunks(a), 256, 0, s>>>(a, a.pairs[from], shift);
    return hipGetLastError();
}

hipError_t launch_embed_scatter(const EmbedGradArgs &a, int from, uint32_t shift, hipStream_t s) {
    if (from < 0) embed_scatter_kernel<true><<<sort_chunks(a), 256, 0, s>>>(a, nullptr, a.pairs[0], shift);
    else embed_scatter_kernel<false><<<sort_chunks(a), 256, 0, s>>>(a, a.pairs[from], a.pairs[1 - from], shift);
    return hipGetLastError();
}

hipError_t launch_embed_sum(int dy, const EmbedGradArgs &a, int sorted, hipStream_t s) {
    const uint32_t units = (a.width + 3) / 4, tx = row_threads(units), rows = 256 / tx;
    const dim3 grid((run_chunks(a) + rows - 1) / rows, (units + tx - 1) / tx);
    if (dy == kF32) embed_sum_kernel<float><<<grid, 256, 0, s>>>(a, a.pairs[sorted], tx);
    else if (dy == kFP16) embed_sum_kernel<_Float16><<<grid, 256, 0, s>>>(a, a.pairs[sorted], tx);
    else embed_sum_kernel<__bf16><<<grid, 256, 0, s>>>(a, a.pairs[sorted], tx);
    return hipGetLastError();
}

hipError_t launch_embed_join(const EmbedGradArgs &a, int sorted, hipStream_t s) {
    const uint32_t tx = row_threads(a.width), rows = 256 / tx;
    embed_join_kernel<<<(run_chunks(a) + rows - 1) / rows, 256, 0, s>>>(a, a.pairs[sorted], tx);
    return hipGetLastError();
}

}  // namespace dedloc
