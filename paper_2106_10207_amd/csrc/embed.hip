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
// A store of what nothing here reads again; the address at any alignment of the element.
template <int N, typename T>
__device__ inline void store_stream(T *p, const float *o) {
    Vec<N, T> q;
#pragma unroll
    for (int i = 0; i < N; i++) q.v[i] = (T)o[i];
    if constexpr (sizeof(q) == 16) {
        typedef unsigned U __attribute__((ext_vector_type(4), aligned(2)));
        __builtin_nontemporal_store(__builtin_bit_cast(U, q), (U *)p);
    } else {
        typedef unsigned U __attribute__((ext_vector_type(2), aligned(2)));
        __builtin_nontemporal_store(__builtin_bit_cast(U, q), (U *)p);
    }
}

// A product rounded to fp32 before it is rounded to 16 bits (without this the
// two become one instruction with one rounding).
__device__ inline float times(float a, float b) {
    float p = a * b;
    asm("" : "+v"(p));
    return p;
}

// Orders what one lane of a wave wrote to LDS before what another reads.
__device__ inline void wave_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// The token at a position; `vocab` for an id outside the table.
__device__ inline uint32_t token(const void *ids, int wide, uint32_t vocab, uint32_t i) {
    const int64_t id = wide ? ((const int64_t *)ids)[i] : (int64_t)((const int32_t *)ids)[i];
    return id >= 0 && id < (int64_t)vocab ? (uint32_t)id : vocab;
}

}  // namespace

// A row of threads (tx of them, a power of two) per position, N elements per
// thread and turn.  Bound by memory once there is enough to move: 131072 x 1024 bf16
// 75 us, 268 MB written and a table of 61 MB read, 4.4 TB/s (as many bytes as are written are loaded, most of them from
// the caches; a plain copy of 2 GB: 5.0), 131072 x 2048 111 to 117 us, 5.2 to 5.5 TB/s, 32768 x 1024 21 us; below 16 MB by the launch, 6 us.  Four positions per row of threads, all loaded before the
// first is stored, took the same times within 3 %.
template <typename TI, typename TO, int N>
__global__ __launch_bounds__(256) void embed_kernel(EmbedArgs a, uint32_t tx) {
    const uint32_t x = threadIdx.x & (tx - 1), rows = 256 / tx;
    const uint64_t row = (uint64_t)blockIdx.x * rows + threadIdx.x / tx;
    if (row >= a.n) return;
    const uint32_t tok = token(a.ids, a.wide_ids, a.vocab, (uint32_t)row);
    const bool named = tok < a.vocab;
    const TI *from = (const TI *)a.table + (uint64_t)tok * a.ld_table;  // read only if named
    TO *to = (TO *)a.out + row * a.ld_out;
    for (uint32_t c = x * N; c < a.width; c += tx * N) {
        if (c + N <= a.width) {
            float v[N] = {};
            if (named) load<N>(from + c, v);
            for (int i = 0; i < N; i++) v[i] = named ? times(v[i], a.scale) : 0.0f;
            store_stream<N>(to + c, v);
        } else {
            for (uint32_t i = c; i < a.width; i++) to[i] = (TO)(named ? times((float)from[i], a.scale) : 0.0f);
        }
    }
}

// ------------------------------------------------------------------ the sort

// One pass orders the positions by a digit of their token, BITS bits, keeping the
// order of equal ones.  Chunk k counts its digits into counts[k][2^BITS].  A pass over 131072 positions takes
// 5.3 us to count and 8.2 to scatter, both near a launch that reads its chunk and the table of counts.
template <bool FIRST>
__device__ inline uint2 pair_at(const EmbedGradArgs &a, const uint2 *from, uint32_t i) {
    if (FIRST) return make_uint2(token(a.ids, a.wide_ids, a.vocab, i), i);
    return from[i];
}

template <bool FIRST, int BITS>
__global__ __launch_bounds__(256) void embed_count_kernel(EmbedGradArgs a, const uint2 *from, uint32_t shift) {
    constexpr uint32_t D = 1u << BITS;
    __shared__ uint32_t count[D];
    for (uint32_t d = threadIdx.x; d < D; d += 256) count[d] = 0;
    __syncthreads();
    const uint32_t i0 = blockIdx.x * a.chunk, i1 = min(i0 + a.chunk, a.n);
    for (uint32_t i = i0 + threadIdx.x; i < i1; i += 256) atomicAdd(&count[(pair_at<FIRST>(a, from, i).x >> shift) & (D - 1)], 1u);
    __syncthreads();
    for (uint32_t d = threadIdx.x; d < D; d += 256) a.counts[blockIdx.x * D + d] = count[d];
}

// The lanes of a wave that have the same digit (of those with `in`).
template <int BITS>
__device__ inline unsigned long long same_digit(uint32_t digit, bool in) {
    unsigned long long same = __ballot(in);
#pragma unroll
    for (int b = 0; b < BITS; b++) {
        const unsigned long long m = __ballot((digit >> b) & 1u);
        same &= (digit >> b) & 1u ? m : ~m;
    }
    return same;
}

// Positions of a wave, 64 a round, in order: an item's rank is how many of the
// wave's items before it have its digit.  at[2^BITS]: the wave's counters, zeroed by
// the caller; afterwards how many items have each digit.
template <uint32_t R, int BITS>
__device__ inline void rank_digits(const uint2 *p, uint32_t left, uint32_t shift, uint32_t *at, uint16_t *rank) {
    const uint32_t lane = threadIdx.x & 63;
#pragma unroll
    for (uint32_t r = 0; r < R; r++) {
        const bool in = r * 64 + lane < left;
        const uint32_t digit = (p[r].x >> shift) & ((1u << BITS) - 1);
        const unsigned long long same = same_digit<BITS>(digit, in);
        const uint32_t mine = __popcll(same & ((1ull << lane) - 1));
        rank[r] = (uint16_t)(at[digit] + mine);
        wave_order();
        if (in && mine == 0) at[digit] += __popcll(same);
        wave_order();
    }
}

// Exclusive sum over threads 0 to 255 of the workgroup (the others pass 0).
__device__ inline uint32_t scan_256(uint32_t v, uint32_t *part) {
    const uint32_t t = threadIdx.x, lane = t & 63, wave = t >> 6;
    uint32_t scan = v;
    for (int off = 1; off < 64; off <<= 1) {
        const uint32_t up = __shfl_up(scan, off, 64);
        if (lane >= (uint32_t)off) scan += up;
    }
    if (wave < 4 && lane == 63) part[wave] = scan;
    __syncthreads();
    for (uint32_t w = 0; w < wave && w < 3; w++) scan += part[w];
    return scan - v;
}

template <bool FIRST, int BITS>
__global__ __launch_bounds__(256) void embed_scatter_kernel(EmbedGradArgs a, const uint2 *from, uint2 *to, uint32_t shift) {
    constexpr uint32_t R = kSortTile / 256, D = 1u << BITS, E = D / 256;
    __shared__ uint32_t at[4][D];  // per wave and digit
    __shared__ uint32_t part[4];
    const uint32_t t = threadIdx.x, lane = t & 63, wave = t >> 6, chunks = gridDim.x;
    // the first places of digits E t on: all smaller digits, and the same digit in the chunks before
    uint32_t before[E] = {}, all[E] = {}, sum = 0;
#pragma unroll 16
    for (uint32_t k = 0; k < chunks; k++)
#pragma unroll
        for (uint32_t e = 0; e < E; e++) {
            const uint32_t c = a.counts[k * D + t * E + e];
            all[e] += c;
            before[e] += k < blockIdx.x ? c : 0;
        }
#pragma unroll
    for (uint32_t e = 0; e < E; e++) sum += all[e];
    uint32_t next = scan_256(sum, part), start[E];
#pragma unroll
    for (uint32_t e = 0; e < E; e++) {
        start[e] = next + before[e];
        next += all[e];
    }
    const uint32_t end = min((blockIdx.x + 1) * a.chunk, a.n);
    for (uint32_t tile = blockIdx.x * a.chunk; tile < end; tile += kSortTile) {
        for (uint32_t d = t; d < 4 * D; d += 256) (&at[0][0])[d] = 0;
        // each wave takes a quarter of the tile, in order
        const uint32_t i0 = tile + wave * (kSortTile / 4), left = i0 < end ? end - i0 : 0;
        uint2 p[R];
        uint16_t rank[R];
#pragma unroll
        for (uint32_t r = 0; r < R; r++)
            p[r] = r * 64 + lane < left ? pair_at<FIRST>(a, from, i0 + r * 64 + lane) : make_uint2(0xffffffffu, 0u);
        __syncthreads();
        rank_digits<R, BITS>(p, left, shift, at[wave], rank);
        __syncthreads();
#pragma unroll
        for (uint32_t e = 0; e < E; e++)
            for (int w = 0; w < 4; w++) {
                const uint32_t c = at[w][t * E + e];
                at[w][t * E + e] = start[e];
                start[e] += c;
            }
        __syncthreads();
#pragma unroll
        for (uint32_t r = 0; r < R; r++)
            if (r * 64 + lane < left) to[at[wave][(p[r].x >> shift) & (D - 1)] + rank[r]] = p[r];
        __syncthreads();
    }
}

// A chunk of 1024 positions sorted by one workgroup, every pass at once, the pairs in
// LDS between the passes: 6.6 us for 8192 positions in two passes of 8 bits, bound by the barriers between their steps.  (All 8192
// in one workgroup took 18.5 us; counting the smaller tokens of each, n^2, 21.6.)
__global__ __launch_bounds__(1024) void embed_sort_kernel(EmbedGradArgs a, uint2 *to) {
    __shared__ uint2 pairs[1024];
    __shared__ uint32_t at[16][256];
    __shared__ uint32_t part[4];
    const uint32_t t = threadIdx.x, wave = t >> 6, i0 = blockIdx.x * 1024, n = min(1024u, a.n - i0);
    const uint32_t left = wave * 64 < n ? n - wave * 64 : 0;
    uint2 p = t < n ? pair_at<true>(a, nullptr, i0 + t) : make_uint2(0xffffffffu, 0u);
    // as many digits as hold `vocab`; a shift of 32 would be one of 0 (a vocab from 2^24 on has all four)
    for (uint32_t shift = 0; shift < 32 && (shift == 0 || a.vocab >> shift); shift += 8) {
        for (uint32_t k = t; k < 16 * 256; k += 1024) (&at[0][0])[k] = 0;
        __syncthreads();
        uint16_t rank;
        rank_digits<1, 8>(&p, left, shift, at[wave], &rank);
        __syncthreads();
        uint32_t c[16], all = 0;
        if (t < 256)
#pragma unroll
            for (int w = 0; w < 16; w++) all += c[w] = at[w][t];
        uint32_t start = scan_256(all, part);
        if (t < 256)
#pragma unroll
            for (int w = 0; w < 16; w++) {
                at[w][t] = start;
                start += c[w];
            }
        __syncthreads();
        if (t < n) pairs[at[wave][(p.x >> shift) & 255u] + rank] = p;
        __syncthreads();
        if (t < n) p = pairs[t];
    }
    if (t < n) to[i0 + t] = p;
}

// Up to kSortOne positions: the sorted chunks merged.  A pair goes to its place in
// its chunk plus, for every other chunk, the number of pairs that come before it, which
// a binary search finds: those of a smaller token, and in earlier chunks those of its own too.
// Eight lanes share a pair's searches; all tokens lie in LDS.  5.5 us for 8192 positions, bound by the reads that
// fill the LDS and the ten dependent steps of a search.
__global__ __launch_bounds__(512) void embed_merge_kernel(EmbedGradArgs a, const uint2 *from, uint2 *to) {
    extern __shared__ __align__(16) uint32_t tok[];
    const uint32_t chunks = (a.n + 1023) / 1024;
#pragma unroll 16
    for (uint32_t k = threadIdx.x * 2; k < chunks * 1024; k += 1024) {
        uint4 p = make_uint4(0xffffffffu, 0u, 0xffffffffu, 0u);
        if (k + 1 < a.n) p = *(const uint4 *)(from + k);
        else if (k < a.n) p.x = from[k].x;
        *(uint2 *)(tok + k) = make_uint2(p.x, p.z);
    }
    __syncthreads();
    const uint32_t i = blockIdx.x * 64 + threadIdx.x / 8, own = i / 1024;
    const uint32_t mine = tok[min(i, a.n - 1)];
    uint32_t place = 0;
    for (uint32_t c0 = threadIdx.x % 8; c0 < chunks; c0 += 16) {
        // in two chunks at a time: the first pair that is not before this one (0 to 1024)
        uint32_t low[2] = {}, limit[2], at[2];
#pragma unroll
        for (uint32_t q = 0; q < 2; q++) {
            const uint32_t c = c0 + 8 * q;
            limit[q] = c < chunks ? mine + (c < own) : 0;  // tokens below it are before; a token is at most 2^30
            at[q] = min(c, chunks - 1) * 1024;
        }
#pragma unroll
        for (uint32_t step = 512; step > 0; step /= 2)
#pragma unroll
            for (uint32_t q = 0; q < 2; q++)
                if (tok[at[q] + low[q] + step - 1] < limit[q]) low[q] += step;
#pragma unroll
        for (uint32_t q = 0; q < 2; q++) {
            low[q] += tok[at[q] + low[q]] < limit[q];
            place += c0 + 8 * q == own ? i % 1024 : low[q];
        }
    }
    for (int off = 1; off < 8; off <<= 1) place += __shfl_xor(place, off, 64);
    if (threadIdx.x % 8 == 0 && i < a.n) to[place] = from[i];
}

// ------------------------------------------------------------------ the sums

// A row of tx threads sums one chunk of a.run sorted positions, N columns per
// thread, kBatch rows of dy (and the accumulator's rows that they end) on their way at a time.  Bound by memory:
// 131072 x 1024 bf16 over 30000 tokens 106 us, 3.8 TB/s of dy and of the accumulator's rows read and written.
constexpr uint32_t kBatch = 4;  // 131072 x 1024 bf16: 2 112 us, 4 107, 8 155

template <typename T, int N>
__global__ __launch_bounds__(256) void embed_sum_kernel(EmbedGradArgs a, const uint2 *pairs, uint32_t tx) {
    const uint32_t x = threadIdx.x & (tx - 1);
    const uint32_t chunk = blockIdx.x * (256 / tx) + threadIdx.x / tx;
    const uint64_t i0 = (uint64_t)chunk * a.run;
    if (i0 >= a.n) return;
    const uint32_t i1 = (uint32_t)(i0 + a.run < a.n ? i0 + a.run : a.n);
    const uint32_t c = (blockIdx.y * tx + x) * N;
    if (c >= a.width) return;
    const bool whole = c + N <= a.width;
    const uint32_t live = whole ? N : a.width - c;
    const T *dy = (const T *)a.dy + c;
    uint32_t tok = i0 > 0 ? pairs[i0 - 1].x : 0xffffffffu;
    bool head = pairs[i0].x == tok;  // the run began in an earlier chunk
    float sum[N] = {};
    for (uint32_t i = (uint32_t)i0; i < i1; i += kBatch) {
        uint2 p[kBatch + 1];
#pragma unroll
        for (uint32_t k = 0; k <= kBatch; k++) p[k] = i + k < a.n ? pairs[i + k] : make_uint2(0xffffffffu, 0u);
        Vec<N, T> v[kBatch];
        float old[kBatch][N];
        // what becomes of row k: nothing (masked, or past the chunk), added, or added as its run's last here
        bool in[kBatch], last[kBatch], cut[kBatch];
        bool began = head;
#pragma unroll
        for (uint32_t k = 0; k < kBatch; k++) {
            in[k] = i + k < i1 && p[k].x < a.vocab;
            const bool more = p[k + 1].x == p[k].x;
            last[k] = in[k] && (!more || i + k + 1 == i1);
            cut[k] = began || (last[k] && more);
            if (last[k]) began = false;
            const T *row = dy + (uint64_t)p[k].y * a.ld_dy;
            const float *acc = a.grad + (uint64_t)p[k].x * a.ld_grad + c;
            if (whole) {
                if (in[k]) v[k] = *(const Vec<N, T> *)row;
                if (last[k] && !cut[k]) load<N>(acc, old[k]);
            } else {
#pragma unroll
                for (uint32_t e = 0; e < N; e++) {
                    v[k].v[e] = e < live && in[k] ? row[e] : (T)0.0f;
                    old[k][e] = e < live && last[k] && !cut[k] ? acc[e] : 0.0f;
                }
            }
        }
#pragma unroll
        for (uint32_t k = 0; k < kBatch; k++) {
            if (!in[k]) continue;
            for (int e = 0; e < N; e++) sum[e] += (float)v[k].v[e];
            if (!last[k]) continue;
            float *to = cut[k] ? a.cut + ((uint64_t)chunk * 2 + (head ? 0 : 1)) * a.width + c
                               : a.grad + (uint64_t)p[k].x * a.ld_grad + c;
            for (int e = 0; e < N; e++) {
                if (!cut[k]) sum[e] = fmaf(a.factor, sum[e], old[k][e]);
            }
            if (whole) store<N>(to, sum);
            else {
#pragma unroll
                for (uint32_t e = 0; e < N; e++)
                    if (e < live) to[e] = sum[e];
            }
            head = false;
            for (int e = 0; e < N; e++) sum[e] = 0.0f;
        }
    }
}

// The runs that leave the chunk they began in: their parts, an equal share of them per wave,
// in ascending order.  A workgroup looks after 256 columns of the run that leaves one
// chunk (four chunks each: 5 us more at 131072 x 1024, 1 us more at 8192 x 128).  Most runs
// have a part or two and cost the workgroup's start and the look ahead; a token that many positions
// share is bound by its few workgroups' loads.
constexpr uint32_t kJoinBatch = 8;  // parts whose loads are on their way at a time

template <uint32_t WAVES>
__global__ __launch_bounds__(64 * WAVES) void embed_join_kernel(EmbedGradArgs a, const uint2 *pairs) {
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, chunks = (a.n + a.run - 1) / a.run;
    const uint32_t c = (blockIdx.y * 64 + lane) * 4, live = c < a.width ? min(4u, a.width - c) : 0;
    __shared__ float part[WAVES][64][4];
    const uint32_t chunk = blockIdx.z * gridDim.x + blockIdx.x;
    const uint64_t i1 = (uint64_t)(chunk + 1) * a.run, i0 = i1 - a.run;
    if (i1 >= a.n) return;
    const uint32_t tok = pairs[i1 - 1].x;
    if (tok >= a.vocab || pairs[i1].x != tok) return;                      // it ends here
    if (i0 > 0 && pairs[i0].x == tok && pairs[i0 - 1].x == tok) return;  // it began earlier
    // the chunks after this one that begin with the run: 64 looked at first, then 512 at a time
    auto begins = [&](uint32_t k) { return k < chunks && pairs[(uint64_t)k * a.run].x == tok; };
    const unsigned long long first = __ballot(begins(chunk + 1 + lane));
    uint32_t more = first == ~0ull ? 64 : (uint32_t)__builtin_ctzll(~first);
    for (bool on = first == ~0ull; on;) {
        bool in[8];
#pragma unroll
        for (uint32_t q = 0; q < 8; q++) in[q] = begins(chunk + 1 + more + q * 64 + lane);
#pragma unroll
        for (uint32_t q = 0; q < 8; q++) {
            const unsigned long long m = __ballot(in[q]);
            if (on) more += m == ~0ull ? 64 : (uint32_t)__builtin_ctzll(~m);
            on = on && m == ~0ull;
        }
    }
    float sum[4] = {};
    if (wave == 0) {
        const float *from = a.cut + ((uint64_t)chunk * 2 + 1) * a.width + c;
#pragma unroll
        for (uint32_t e = 0; e < 4; e++)
            if (e < live) sum[e] = from[e];
    }
    const uint32_t k1 = chunk + 1 + (uint32_t)((uint64_t)more * (wave + 1) / WAVES);
    uint32_t k = chunk + 1 + (uint32_t)((uint64_t)more * wave / WAVES);
    for (; k < k1; k += kJoinBatch) {
        float v[kJoinBatch][4] = {};
#pragma unroll
        for (uint32_t b = 0; b < kJoinBatch; b++) {
            const float *from = a.cut + (uint64_t)(k + b) * 2 * a.width + c;
            if (k + b < k1 && live == 4) load<4>(from, v[b]);
            if (k + b < k1 && live < 4)
#pragma unroll
                for (uint32_t e = 0; e < 3; e++)
                    if (e < live) v[b][e] = from[e];
        }
#pragma unroll
        for (uint32_t b = 0; b < kJoinBatch; b++)
            for (int e = 0; e < 4; e++) sum[e] += v[b][e];
    }
    for (int e = 0; e < 4; e++) part[wave][lane][e] = sum[e];
    __syncthreads();
    if (wave > 0) return;
    for (uint32_t w = 1; w < WAVES; w++)
        for (int e = 0; e < 4; e++) sum[e] += part[w][lane][e];
    float *to = a.grad + (uint64_t)tok * a.ld_grad + c;
#pragma unroll
    for (uint32_t e = 0; e < 4; e++)
        if (e < live) to[e] = fmaf(a.factor, sum[e], to[e]);
}

// ---------------------------------------------------------------- launchers

namespace {

constexpr uint32_t kGridMost = 1u << 23;  // workgroups along one side of a grid: 2^32 threads are too many

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
    const uint64_t most = (uint64_t)kGridMost * rows;  // positions of a launch
    for (uint64_t i = 0; i < a.n; i += most) {
        EmbedArgs b = a;
        b.ids = (const char *)a.ids + i * (a.wide_ids ? 8 : 4);
        b.out = (TO *)a.out + i * a.ld_out;
        b.n = (uint32_t)std::min(a.n - i, most);
        embed_kernel<TI, TO, N><<<(b.n + rows - 1) / rows, 256, 0, s>>>(b, tx);
    }
}
template <typename TI>
void embed(int out, const EmbedArgs &a, hipStream_t s) {
    if (out == kF32) embed<TI, float>(a, s);
    else if (out == kFP16) embed<TI, _Float16>(a, s);
    else embed<TI, __bf16>(a, s);
}

uint32_t sort_chunks(const EmbedGradArgs &a) { return (a.n + a.chunk - 1) / a.chunk; }
uint32_t run_chunks(const EmbedGradArgs &a) { return (a.n + a.run - 1) / a.run; }

template <typename T>
void sum(const EmbedGradArgs &a, const uint2 *pairs, hipStream_t s) {
    constexpr int N = 16 / sizeof(T);
    const uint32_t units = (a.width + N - 1) / N, tx = row_threads(units), rows = 256 / tx;
    const dim3 grid((run_chunks(a) + rows - 1) / rows, (units + tx - 1) / tx);
    embed_sum_kernel<T, N><<<grid, 256, 0, s>>>(a, pairs, tx);
}

}  // namespace

hipError_t launch_embed(int table, int out, const EmbedArgs &a, hipStream_t s) {
    if (table == kF32) embed<float>(out, a, s);
    else if (table == kFP16) embed<_Float16>(out, a, s);
    else embed<__bf16>(out, a, s);
    return hipGetLastError();
}

namespace {
template <int BITS>
void count(const EmbedGradArgs &a, int from, uint32_t shift, hipStream_t s) {
    if (from < 0) embed_count_kernel<true, BITS><<<sort_chunks(a), 256, 0, s>>>(a, nullptr, shift);
    else embed_count_kernel<false, BITS><<<sort_chunks(a), 256, 0, s>>>(a, a.pairs[from], shift);
}
template <int BITS>
void scatter(const EmbedGradArgs &a, int from, uint32_t shift, hipStream_t s) {
    if (from < 0) embed_scatter_kernel<true, BITS><<<sort_chunks(a), 256, 0, s>>>(a, nullptr, a.pairs[0], shift);
    else embed_scatter_kernel<false, BITS><<<sort_chunks(a), 256, 0, s>>>(a, a.pairs[from], a.pairs[1 - from], shift);
}
}  // namespace

hipError_t launch_embed_count(const EmbedGradArgs &a, int from, uint32_t bits, uint32_t shift, hipStream_t s) {
    if (bits <= 8) count<8>(a, from, shift, s);
    else if (bits == 9) count<9>(a, from, shift, s);
    else count<kSortBits>(a, from, shift, s);
    return hipGetLastError();
}

hipError_t launch_embed_scatter(const EmbedGradArgs &a, int from, uint32_t bits, uint32_t shift, hipStream_t s) {
    if (bits <= 8) scatter<8>(a, from, shift, s);
    else if (bits == 9) scatter<9>(a, from, shift, s);
    else scatter<kSortBits>(a, from, shift, s);
    return hipGetLastError();
}

hipError_t launch_embed_sort(const EmbedGradArgs &a, hipStream_t s) {
    embed_sort_kernel<<<(a.n + 1023) / 1024, 1024, 0, s>>>(a, a.pairs[0]);
    return hipGetLastError();
}

hipError_t launch_embed_merge(const EmbedGradArgs &a, hipStream_t s) {
    const uint32_t bytes = (a.n + 1023) / 1024 * 4096;
    embed_merge_kernel<<<(a.n + 63) / 64, 512, bytes, s>>>(a, a.pairs[0], a.pairs[1]);
    return hipGetLastError();
}

hipError_t launch_embed_sum(int dy, const EmbedGradArgs &a, int sorted, hipStream_t s) {
    if (dy == kF32) sum<float>(a, a.pairs[sorted], s);
    else if (dy == kFP16) sum<_Float16>(a, a.pairs[sorted], s);
    else sum<__bf16>(a, a.pairs[sorted], s);
    return hipGetLastError();
}

hipError_t launch_embed_join(const EmbedGradArgs &a, int sorted, hipStream_t s) {
    const uint32_t chunks = run_chunks(a), x = std::min(chunks, kGridMost);
    const dim3 grid(x, (a.width + 255) / 256, (chunks + x - 1) / x);
    // 8 or 4 waves, the whole gradient, us: with tokens at random 21.3, 21.2 (8192 x 128, 1024 workgroups), 42, 41 (16384 x 768,
    // 3 x 1024), 183, 168 (131072 x 1024, 16384); with half of the positions one token 30, 36, 48, 52 and 222, 231
    if ((uint64_t)chunks * grid.y <= 4096) embed_join_kernel<8><<<grid, 512, 0, s>>>(a, a.pairs[sorted]);
    else embed_join_kernel<4><<<grid, 256, 0, s>>>(a, a.pairs[sorted]);
    return hipGetLastError();
}

}  // namespace dedloc
