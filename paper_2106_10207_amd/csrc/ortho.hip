// gfx950 kernels of the orthogonalised update (Newton-Schulz steps) and the
// Muon step built on it.
//
// With s the shorter side of a matrix and l the longer, X [s][l] is taken
// towards the nearest matrix with orthogonal rows by
//   X0 = G / (|G|_F + eps),   A = X X^T,   M = a I + b A + c A^2,   X <- M X.
// Everything that multiplies X is a polynomial of A, symmetric, and commutes, so
// n steps can be taken on the s x s side, A <- M A M, with one Gram matrix before
// them and one product Q X, Q = M_n ... M_1, after: 3 s^2 l + (4 n - 3) s^3 multiply-adds
// for n (3 s^2 l + s^3), symmetric products counted half.
//
// Precision.  A singular value far below 1 grows by a (3.4) in a step, and a
// rounding error of X with it, so five steps multiply it by up to a^5 = 485:
// operands of 11 bits (fp16) lose 1e-2 of the result of an ill-conditioned
// gradient, 8 bits (bf16) 1e-1.  So every operand is held in two fp16 planes,
// hi + lo, 22 bits, and a product takes three of them,
//   hi hi' + hi lo' + lo hi'
// in fp32 accumulators.  An error of A grows by a^2 in a step on the s x s side: three
// steps from X0 and two from later X keep it small; five lose it altogether.  Fine results (fp32, and the
// update of Muon's fp32 parameters) also round their sums every two turns and take lo lo' where sums are
// short; orthogonalize's leave long matrices out of the blocks: errors of 3e-7 to 2e-6 of the result, about half
// of those of fp32 products.
// X is stored times 2^12, the symmetric matrices times 2^8: |X| stays below 1.3 and
// |Q| below a^3 = 41, and the low planes of entries of the usual size (1 / sqrt(s l))
// stay in fp16's normal range.
//
// Layout of a two-plane matrix: panels of 32 columns, in a panel the rows one after
// the other, 128 bytes each, 64 of hi then 64 of lo.  A turn of a product's loop
// reads a tile's rows of one panel, one piece of memory.  (Row by row, the rows
// of a tile would lie 4 l bytes apart, for most matrices a power of two, and so
// on one of the L2's channels.)
// Both factors of every product have the summed index along their rows: the
// small matrices are symmetric, and X^T is kept beside X.
#include <algorithm>
#include <type_traits>

#include "ops_internal.h"

namespace dedloc {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

namespace {

// An fp32 result, and Muon's step of fp32 parameters, keeps what its type holds: sums that no truncation biases and,
// where they have few terms (a shorter side up to kFourProducts), lo lo' too.  Of Muon's update this takes 1 to
// 2.5 % more time (ALBERT-large 907 us for 894, ResNet-50's matrices 1013 for 1003, ALBERT-xlarge 4998 for 4880) and
// halves its error: 1.4e-6 to 1.7e-6 for 2.8e-6 to 4.0e-6, in plain fp32 products 2.7e-6 to 3.2e-6.
template <int OUT>
constexpr bool kFine = OUT == kNsF32 || OUT == kNsMuonF32;
constexpr uint32_t kFourProducts = 64;

constexpr float kXScale = 4096.0f;  // of X
constexpr float kAScale = 256.0f;   // of the symmetric matrices

struct Sides {
    uint32_t s, l, S, L;
    bool tall;  // rows > cols: X is the transpose
};
__device__ inline Sides sides(uint32_t rows, uint32_t cols) {
    Sides d;
    d.tall = rows > cols;
    d.s = d.tall ? cols : rows;
    d.l = d.tall ? rows : cols;
    d.S = (d.s + kNsPad - 1) / kNsPad * kNsPad;
    d.L = (d.l + kNsPad - 1) / kNsPad * kNsPad;
    return d;
}

// A buffer of a matrix' region.
__device__ inline char *buffer(const NsArgs &a, uint64_t base, const Sides &d, uint32_t k) {
    const uint64_t big = (uint64_t)d.S * d.L * 4, small = (uint64_t)d.S * d.S * 4;
    return a.ws + base + (k < kNsSmall ? k * big : kNsSmall * big + (k - kNsSmall) * small);
}
// Byte offset of element (i, j) of a matrix of `rows` rows: its hi; lo is 64 bytes on.
__device__ inline uint64_t at_planes(uint32_t i, uint32_t j, uint32_t rows) {
    return ((uint64_t)(j / 32) * rows + i) * 128 + (j % 32) * 2;
}

__device__ inline void split(float v, _Float16 &hi, _Float16 &lo) {
    hi = (_Float16)v;
    lo = (_Float16)(v - (float)hi);
}

// The entry of a table that workgroup `wg` belongs to: the last that begins at or before it.  The lanes
// look at an entry each (one entry after the other: 135 us instead of 122 for 8 matrices of 256 x 512).
template <typename T>
__device__ inline uint32_t find(const T *m, uint32_t n, uint32_t wg) {
    static_assert(kNsWorks <= 128, "");
    const uint32_t lane = threadIdx.x & 63;
    uint32_t k = __popcll(__ballot(lane < n && m[lane].begin <= wg));
    if (n > 64) k += __popcll(__ballot(lane + 64 < n && m[lane + 64].begin <= wg));
    return k - 1;
}

// Entry `e` (flat, absolute) of an averaged gradient.
template <int SRC>
__device__ inline float grad_at(const NsArgs &a, uint64_t e) {
    if (SRC == kNsMuonF32) return ((const float *)a.grad)[e];
    if (SRC == kNsMuonFP16) return (float)((const _Float16 *)a.grad)[e];
    return (float)((const int8_t *)a.grad)[e] * a.scales[e >> 10];
}

// Four of them; e is a multiple of 4, so they share a block of the int8 codec.
template <int SRC>
__device__ inline void grads_at(const NsArgs &a, uint64_t e, float *g) {
    if constexpr (SRC == kNsMuonF32) {
        *(f32x4 *)g = *(const f32x4 *)((const float *)a.grad + e);
    } else if constexpr (SRC == kNsMuonFP16) {
        const f16x4 v = *(const f16x4 *)((const _Float16 *)a.grad + e);
        for (int q = 0; q < 4; q++) g[q] = (float)v[q];
    } else {
        typedef int8_t i8x4 __attribute__((ext_vector_type(4)));
        const i8x4 v = *(const i8x4 *)((const int8_t *)a.grad + e);
        const float scale = a.scales[e >> 10];
        for (int q = 0; q < 4; q++) g[q] = (float)v[q] * scale;
    }
}

template <int SRC>
__device__ inline float entry(const NsArgs &a, const NsMat &m, uint32_t row, uint32_t col) {
    if (SRC >= kNsMuonF32) {
        const uint64_t e = m.ld_in + (uint64_t)row * m.cols + col;
        const float mom = a.mom[e];
        return a.nesterov ? fmaf(a.mu, mom, grad_at<SRC>(a, e)) : mom;
    }
    const uint64_t e = (uint64_t)row * m.ld_in + col;
    if (SRC == kNsF32) return ((const float *)m.in)[e];
    if (SRC == kNsFP16) return (float)((const _Float16 *)m.in)[e];
    return (float)((const __bf16 *)m.in)[e];
}

__device__ inline double block_sum(double v) {
    __shared__ double red[4];
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = (red[0] + red[1]) + (red[2] + red[3]);
    __syncthreads();
    return v;
}

}  // namespace

// A thread's entries of the block of kNsTile rows and columns at (r0, c0): column threadIdx.x % 64,
// rows threadIdx.x / 64 + 4 k.  All loads are on their way before the first is used.
constexpr uint32_t kBlockEntries = kNsTile * kNsTile / 256;
template <int SRC>
__device__ inline void block_entries(const NsArgs &a, const NsMat &m, uint32_t r0, uint32_t c0, float *v) {
    const uint32_t row = r0 + threadIdx.x / kNsTile, col = c0 + threadIdx.x % kNsTile;
#pragma unroll
    for (uint32_t k = 0; k < kBlockEntries; k++)
        v[k] = row + 4 * k < m.rows && col < m.cols ? entry<SRC>(a, m, row + 4 * k, col) : 0.0f;
}

// Sums of squares in 64 bits, each of every kSumMost-th block of kNsTile rows and
// columns: one block for most matrices.  13.8M fp32 elements of 8 matrices 25 us, 2.2 TB/s;
// blocks of 16 x 256 took as long.
template <int SRC, int N>
__global__ __launch_bounds__(256) void ns_sum_kernel(NsMats<N> t, NsArgs a) {
    const NsMat &m = t.m[find(t.m, t.n, blockIdx.x)];
    const uint32_t k = blockIdx.x - m.begin, across = (m.cols + kNsTile - 1) / kNsTile;
    const uint32_t blocks = across * ((m.rows + kNsTile - 1) / kNsTile);
    double sum = 0.0;
    for (uint32_t b = k; b < blocks; b += kSumMost) {
        float v[kBlockEntries];
        block_entries<SRC>(a, m, b / across * kNsTile, b % across * kNsTile, v);
#pragma unroll
        for (uint32_t i = 0; i < kBlockEntries; i++) sum = fma((double)v[i], (double)v[i], sum);
    }
    sum = block_sum(sum);
    if (threadIdx.x == 0) a.part[m.part + k] = sum;
}

// Muon: m' = fma(mu, m, g), and the sums of squares of the update, each of every
// kSumMost-th chunk of kSumChunk elements.  Bound by memory: 54.8M elements with an int8
// gradient (9 bytes each) 75 us, 6.6 TB/s.
template <int SRC, int N>
__global__ __launch_bounds__(256) void muon_sum_kernel(NsMats<N> t, NsArgs a) {
    const NsMat &m = t.m[find(t.m, t.n, blockIdx.x)];
    const uint32_t k = blockIdx.x - m.begin;
    const uint64_t n = (uint64_t)m.rows * m.cols;
    double sum = 0.0;
    for (uint64_t i0 = (uint64_t)k * kSumChunk; i0 < n; i0 += (uint64_t)kSumMost * kSumChunk) {
        const uint64_t end = min(i0 + kSumChunk, n);
        for (uint64_t i = i0 + threadIdx.x * 4; i < end; i += 256 * 4) {
            const uint64_t e = m.ld_in + i;  // a multiple of 4
            alignas(16) float g[4], mom[4];
            const bool whole = i + 4 <= end;
            if (whole) {
                grads_at<SRC>(a, e, g);
                *(f32x4 *)mom = *(const f32x4 *)(a.mom + e);
            } else {
                for (uint32_t q = 0; q < 4; q++) {
                    g[q] = i + q < end ? grad_at<SRC>(a, e + q) : 0.0f;
                    mom[q] = i + q < end ? a.mom[e + q] : 0.0f;
                }
            }
#pragma unroll
            for (uint32_t q = 0; q < 4; q++) {
                mom[q] = fmaf(a.mu, mom[q], g[q]);
                const double u = a.nesterov ? fmaf(a.mu, mom[q], g[q]) : mom[q];
                sum = fma(u, u, sum);
            }
            if (whole) *(f32x4 *)(a.mom + e) = *(const f32x4 *)mom;
            else
                for (uint32_t q = 0; q < 4; q++)
                    if (i + q < end) a.mom[e + q] = mom[q];
        }
    }
    sum = block_sum(sum);
    if (threadIdx.x == 0) a.part[m.part + k] = sum;
}

// X0 and its transpose in two planes, zeros in the padding: one workgroup per
// block of 64 x 64 of the matrix as it is stored.  Bound by memory: the same elements
// (12 bytes each without Nesterov's momentum) 127 us, 5.2 TB/s.
template <int SRC, int N>
__global__ __launch_bounds__(256) void ns_prepare_kernel(NsMats<N> t, NsArgs a) {
    const uint32_t q = find(t.m, t.n, blockIdx.x);
    const NsMat &m = t.m[q];
    const Sides d = sides(m.rows, m.cols);
    const uint32_t k = blockIdx.x - m.begin;
    const uint32_t across = (d.tall ? d.S : d.L) / 64, r0 = k / across * 64, c0 = k % across * 64;
    float v[kBlockEntries];
    block_entries<SRC>(a, m, r0, c0, v);
    double sum = 0.0;
    const uint32_t end = q + 1 < t.n ? t.m[q + 1].part : t.parts;
    for (uint32_t i = m.part + threadIdx.x; i < end; i += 256) sum += a.part[i];
    sum = block_sum(sum);
    // in 64 bits: of fp32's smallest numbers, or its largest, the factor is not one of fp32's; and zeros stay zeros if eps is 0
    const double scale = sum == 0.0 ? 0.0 : (double)kXScale / (sqrt(sum) + (double)a.eps);
    __shared__ float tile[64][65];
#pragma unroll
    for (uint32_t i = 0; i < kBlockEntries; i++) tile[threadIdx.x / 64 + 4 * i][threadIdx.x % 64] = (float)((double)v[i] * scale);
    __syncthreads();
    // The block as stored goes to X (wide) or X^T (tall), its transpose to the other, 8 entries of a row
    // at a time: 16 bytes of each plane, from 64 banks.
    char *straight = buffer(a, m.base, d, d.tall), *turned = buffer(a, m.base, d, !d.tall);
    const uint32_t h_straight = d.tall ? d.L : d.S, h_turned = d.tall ? d.S : d.L;
    const uint32_t e0 = threadIdx.x % 8 * 8;
#pragma unroll
    for (uint32_t r = threadIdx.x / 8; r < 64; r += 32) {
        f16x8 hi, lo;
#pragma unroll
        for (uint32_t e = 0; e < 8; e++) {
            _Float16 h, w;
            split(tile[r][e0 + e], h, w);
            hi[e] = h;
            lo[e] = w;
        }
        char *p = straight + at_planes(r0 + r, c0 + e0, h_straight);
        *(f16x8 *)p = hi;
        *(f16x8 *)(p + 64) = lo;
#pragma unroll
        for (uint32_t e = 0; e < 8; e++) {
            _Float16 h, w;
            split(tile[e0 + e][r], h, w);
            hi[e] = h;
            lo[e] = w;
        }
        p = turned + at_planes(c0 + r, r0 + e0, h_turned);
        *(f16x8 *)p = hi;
        *(f16x8 *)(p + 64) = lo;
    }
}

// An entry of a I + b A + c A^2, all times kAScale.  In 64 bits: where A is near 1 the terms are nine times
// their sum.
__device__ inline float polynomial(const NsArgs &a, float A, double A2, bool diagonal) {
    return (float)fma((double)a.b, (double)A, fma((double)a.c, A2, diagonal ? (double)a.a * (double)kAScale : 0.0));
}

// Orders what one lane of a wave wrote to LDS before what another reads.
__device__ inline void wave_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

template <int N, typename T>
struct Vec {
    T v[N];
} __attribute__((packed, aligned(sizeof(T))));

constexpr uint32_t kTurnPitch = 36;  // words of a row of a block that is turned in LDS

// A block of the call's result: the lane's row is i of X; acc[4 g + e] belongs to
// column j0 + 8 g + 4 (lane / 32) + e.
template <int OUT>
__device__ inline void ns_result(const NsWork &m, const Sides &d, const NsArgs &a, uint32_t i, uint32_t j0, const f32x16 &acc) {
    const uint32_t lane = threadIdx.x & 63;
    if (i >= d.s) return;
    const uint64_t ld = OUT == kNsMuonF32 ? m.cols : m.ld_out;
    const uint64_t step = d.tall ? ld : 1;  // from column j to the next
#pragma unroll
    for (uint32_t g = 0; g < 4; g++) {
        const uint32_t j = j0 + 8 * g + 4 * (lane / 32);
        if (j >= d.l) break;
        const uint32_t n = min(4u, d.l - j);
        const uint64_t at = d.tall ? j * ld + i : i * ld + j;
        float v[4];
        for (int e = 0; e < 4; e++) v[e] = acc[4 * g + e] * (1.0f / (kAScale * kXScale));
        if constexpr (OUT == kNsMuonF32) {
            float *x = a.x + m.ld_out + at;
            const float keep = (m.op >> 16 & 1) ? a.keep : 1.0f;
            if (!d.tall && n == 4) {
                Vec<4, float> q = *(const Vec<4, float> *)x;
                for (int e = 0; e < 4; e++) q.v[e] = fmaf(-m.unit, v[e], keep * q.v[e]);
                *(Vec<4, float> *)x = q;
            } else {
                for (uint32_t e = 0; e < n; e++) x[e * step] = fmaf(-m.unit, v[e], keep * x[e * step]);
            }
        } else {
            typedef std::conditional_t<OUT == kNsF32, float, std::conditional_t<OUT == kNsFP16, _Float16, __bf16>> T;
            T *to = (T *)m.out + at;
            if (!d.tall && n == 4) {
                Vec<4, T> q;
                for (int e = 0; e < 4; e++) q.v[e] = (T)v[e];
                *(Vec<4, T> *)to = q;
            } else {
                for (uint32_t e = 0; e < n; e++) to[e * step] = (T)v[e];
            }
        }
    }
}

// What a block of 32 x 32 (rows i0, columns j0 on) of a product becomes.  The lane's
// row is i = i0 + lane % 32; acc[4 g + e] belongs to column j0 + 8 g + 4 (lane / 32) + e.
// turn: 32 * kTurnPitch words of the wave's own in LDS, through which the block goes
// to its transposed place in whole pieces of 32 bytes.
template <int OUT>
__device__ inline void ns_finish(const NsWork &m, const Sides &d, const NsArgs &a, uint32_t i0, uint32_t j0, const f32x16 &acc,
                                 uint32_t *turn) {
    const uint32_t lane = threadIdx.x & 63, il = lane % 32, i = i0 + il, kind = m.op & 15;
    if (kind == kNsResult) return ns_result<OUT>(m, d, a, i, j0, acc);
    const float scale = kind == kNsGram ? kAScale / (kXScale * kXScale) : 1.0f / kAScale;
    char *to = buffer(a, m.base, d, kind == kNsApply ? 0 : m.op >> 12 & 15) + at_planes(i, j0, d.S);
    const char *old = buffer(a, m.base, d, m.op >> 4 & 15) + at_planes(i, j0, d.S);
    wave_order();  // the block before has left `turn`
#pragma unroll
    for (uint32_t g = 0; g < 4; g++) {
        const uint32_t jl = 8 * g + 4 * (lane / 32);
        float v[4];
        f16x4 hi, lo;
        for (int e = 0; e < 4; e++) v[e] = acc[4 * g + e] * scale;
        if (kind == kNsSquare) {
            hi = *(const f16x4 *)(old + jl * 2);
            lo = *(const f16x4 *)(old + jl * 2 + 64);
            for (int e = 0; e < 4; e++)
                v[e] = polynomial(a, (float)hi[e] + (float)lo[e], v[e], i == j0 + jl + e);
        }
        for (int e = 0; e < 4; e++) {
            _Float16 h, w;
            split(v[e], h, w);
            hi[e] = h;
            lo[e] = w;
            turn[(jl + e) * kTurnPitch + il] = (uint32_t)__builtin_bit_cast(uint16_t, h) | (uint32_t)__builtin_bit_cast(uint16_t, w) << 16;
        }
        *(f16x4 *)(to + jl * 2) = hi;
        *(f16x4 *)(to + jl * 2 + 64) = lo;
    }
    if (kind != kNsApply && i0 == j0) return;
    // the transpose: X^T, or the upper triangle.  The lane has row j0 + lane % 32 and 16 of its columns.
    wave_order();
    u32x4 q[4];
#pragma unroll
    for (uint32_t k = 0; k < 4; k++) q[k] = *(const u32x4 *)(turn + il * kTurnPitch + 16 * (lane / 32) + 4 * k);
    to = buffer(a, m.base, d, m.op >> 12 & 15) + at_planes(j0 + il, i0 + 16 * (lane / 32), kind == kNsApply ? d.L : d.S);
#pragma unroll
    for (uint32_t k = 0; k < 2; k++) {
        u32x4 hi, lo;
#pragma unroll
        for (uint32_t w = 0; w < 4; w++) {
            const uint32_t x = q[2 * k + w / 2][w % 2 * 2], y = q[2 * k + w / 2][w % 2 * 2 + 1];
            hi[w] = (x & 0xffffu) | y << 16;
            lo[w] = x >> 16 | (y & 0xffff0000u);
        }
        *(u32x4 *)(to + 16 * k) = hi;
        *(u32x4 *)(to + 64 + 16 * k) = lo;
    }
}

// The tile of a product's work item: tiles of the same piece of the summed index
// follow one another.
struct Tile {
    uint32_t ti, tj, piece, tiles;
};
__device__ inline Tile tile_at(const NsWork &m, const Sides &d, uint32_t k, uint32_t T) {
    Tile t;
    const uint32_t down = (d.S + T - 1) / T, across = (d.L + T - 1) / T;
    const bool full = (m.op & 15) >= kNsApply;
    t.tiles = full ? down * across : down * (down + 1) / 2;
    t.piece = k / t.tiles;
    k %= t.tiles;
    if (full) {
        // bands of 8 tile rows, column by column: a tile's neighbours in time share its factors
        const uint32_t band = k / (8 * across), high = min(8u, down - band * 8);
        k -= band * 8 * across;
        t.ti = band * 8 + k % high;
        t.tj = k / high;
    } else {  // the lower triangle of a symmetric result
        uint32_t u = (uint32_t)((sqrtf(8.0f * k + 1.0f) - 1.0f) * 0.5f);
        while ((u + 1) * (u + 2) / 2 <= k) u++;
        while (u * (u + 1) / 2 > k) u--;
        t.ti = u;
        t.tj = k - u * (u + 1) / 2;
    }
    return t;
}

// The summed index of a work's products, in elements.
__device__ inline uint32_t summed(const NsWork &m) {
    const Sides d = sides(m.rows, m.cols);
    return (m.op & 15) == kNsGram ? d.L : d.S;
}

// The item of this workgroup.  Workgroups go round the 8 XCDs; of the works with the same
// summed index, which follow one another in the table, the longest first, each XCD gets a contiguous
// range of items, as many as the others.  (One range of all works for each: the first XCDs had the long
// sums, 1269 us instead of 1090 for the 54 matrices of a ResNet-50.)
template <int N>
__device__ inline uint32_t item_of(const NsList<N> &t) {
    uint32_t begin = 0, end = gridDim.x;
    if (t.mixed) {
        const uint32_t lane = threadIdx.x & 63, mine = summed(t.w[find(t.w, t.n, blockIdx.x)]);
        uint32_t first = 0, same = 0;
#pragma unroll
        for (uint32_t q = 0; q < N; q += 64) {
            const bool in = q + lane < t.n;
            const uint32_t K = in ? summed(t.w[q + lane]) : 0;
            first += __popcll(__ballot(in && K > mine));
            same += __popcll(__ballot(in && K == mine));
        }
        begin = t.w[first].begin;
        if (first + same < t.n) end = t.w[first + same].begin;
    }
    const uint32_t at = blockIdx.x - begin, n = end - begin;
    return begin + at % 8 * (n / 8) + min(at % 8, n % 8) + at / 8;
}

typedef __attribute__((address_space(3))) void *LdsPtr;

// Waits until at most N of this wave's loads are in flight and its LDS reads are done, then for the workgroup's other
// waves.  (A fence would wait for LDS alone, __syncthreads for every load.)
template <int N>
__device__ inline void arrived() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4 << 14) | 0x70);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}
constexpr int kRawBuffer = 0x00020000;  // descriptor of untyped bytes
constexpr int kSchedMfma = 0x8, kSchedLoad = 0x10, kSchedRead = 0x100;  // classes of sched_group_barrier

// A shape of tile: `edge` rows and columns, wi x wj blocks of 32 x 32 per wave, two
// waves to a row of them.  Two workgroups of either kind fit a CU (64 KB of LDS
// each, the big ones 65: the two stages that they lack are 16 bytes, aligned to 1024): big tiles with one turn of loads in flight beside the one worked on, little ones, whose
// turns are short, with three.
template <uint32_t EDGE, uint32_t WI, uint32_t WJ, uint32_t STAGES, uint32_t PER_SIMD>
struct Shape {
    static constexpr uint32_t edge = EDGE, wi = WI, wj = WJ, waves = EDGE / 32 * EDGE / 32 / (WI * WJ), stages = STAGES,
                              per_simd = PER_SIMD;
};
typedef Shape<128, 2, 2, 2, 2> Big;
typedef Shape<64, 1, 1, 4, 2> Little;

// One tile of a product of a step over a piece of the summed index.  OUT: the dtype of a result, or
// kNsMuonF32 for the update of the parameters.
//
// A turn of the loop takes 32 of the summed index, 128 bytes of a row of either
// factor.  They go from memory into one of NS stages of LDS without passing
// registers, NS - 1 turns ahead, and from there into registers half a turn ahead, so that
// the matrix cores find their operands; loads and reads are dealt out between the products.
// 16-byte piece c of row r lies at place c ^ (r / 2 % 8) of its row, so that 16
// lanes of a read, one row each, meet all 64 banks (with r % 8 two rows met in a bank
// and every read took 8 cycles instead of 4); the load writes lanes in order, so
// the lane picks its source piece instead.
//
// Large products are bound by the card's power: those of 8 matrices up to 8192 x 2048 (17 launches, 4.81 ms)
// run at 0.94 PFLOP/s, three fp16 products for one, the clock between 1.75 and 1.9 GHz (these instructions alone, on random operands, reach
// 1.6 to 1.7 PFLOP/s, with the loop's loads and reads 1.40; a large library product of fp16 1.20).
// Small ones are bound by the launch: 4.5 us, and 5.3 for tiles of 64 with 4 turns.
template <int OUT, typename C, int N>
__global__ __launch_bounds__(64 * C::waves, C::per_simd) void ns_product_kernel(NsList<N> t, NsArgs a) {
    constexpr uint32_t T = C::edge, NW = C::waves, WI = C::wi, WJ = C::wj, NS = C::stages;
    const uint32_t wg = item_of(t);
    const NsWork &m = t.w[find(t.w, t.n, wg)];
    const Sides d = sides(m.rows, m.cols);
    const Tile tile = tile_at(m, d, wg - m.begin, T);
    const uint32_t i0 = tile.ti * T, j0 = tile.tj * T, kind = m.op & 15;
    const uint32_t K = summed(m);
    const char *left = buffer(a, m.base, d, m.op >> 4 & 15), *right = buffer(a, m.base, d, m.op >> 8 & 15);
    const uint32_t left_rows = d.S, right_rows = kind >= kNsApply ? d.L : d.S;

    constexpr uint32_t kStage = 2 * T * 128;
    // one array per stage: the compiler then knows which loads a read has to wait for
    __shared__ __align__(1024) char lds0[kStage], lds1[NS > 1 ? kStage : 16], lds2[NS > 2 ? kStage : 16],
        lds3[NS > 3 ? kStage : 16];
    auto stage = [&](uint32_t k) { return k == 0 ? lds0 : k == 1 ? lds1 : k == 2 ? lds2 : lds3; };
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t wi = wave / 2 * (32 * WI), wj = wave % 2 * (32 * WJ);
    // A load of a wave takes 8 rows.  The panels' rows past the matrix' end lie beyond the descriptor's end and read as 0.
    constexpr uint32_t kLoads = 2 * T / 8 / NW;
    const uint32_t from = wave * 1024 + (lane / 8) * 128 + ((lane % 8) ^ ((wave % 2) * 4 + lane / 16)) * 16;
    const uint64_t left_panel = (uint64_t)left_rows * 128, right_panel = (uint64_t)right_rows * 128;
    const uint32_t left_end = min(left_rows - i0, T) * 128, right_end = min(right_rows - j0, T) * 128;
    const uint32_t first = (uint64_t)(K / 32) * tile.piece / m.pieces;
    const uint32_t panels = (uint32_t)((uint64_t)(K / 32) * (tile.piece + 1) / m.pieces) - first;
    left += (uint64_t)i0 * 128 + first * left_panel;
    right += (uint64_t)j0 * 128 + first * right_panel;
    auto fetch = [&](char *lds, uint32_t panel) {
        const uint64_t p = min(panel, panels - 1);  // past the end the last once more: the loop then counts its loads
        const auto lrows = __builtin_amdgcn_make_buffer_rsrc((void *)(left + p * left_panel), 0, left_end, kRawBuffer);
        const auto rrows = __builtin_amdgcn_make_buffer_rsrc((void *)(right + p * right_panel), 0, right_end, kRawBuffer);
#pragma unroll
        for (uint32_t q = 0; q < kLoads; q++)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(q < kLoads / 2 ? lrows : rrows, (LdsPtr)(lds + (q * NW + wave) * 1024), 16,
                                                     from, q % (kLoads / 2) * NW * 1024, 0, 0);
    };
    f32x16 acc[WI][WJ] = {};
    f16x8 l[2][WI][2], r[2][WJ][2];  // [half of the turn][block][plane]
    auto read = [&](const char *lds, uint32_t h) {
        auto one = [&](uint32_t row, uint32_t p) {
            const uint32_t c = p * 4 + h * 2 + lane / 32;
            return *(const f16x8 *)(lds + row * 128 + ((c ^ (row / 2 % 8)) * 16));
        };
#pragma unroll
        for (uint32_t p = 0; p < 2; p++) {
#pragma unroll
            for (uint32_t b = 0; b < WI; b++) l[h][b][p] = one(wi + b * 32 + lane % 32, p);
#pragma unroll
            for (uint32_t b = 0; b < WJ; b++) r[h][b][p] = one(T + wj + b * 32 + lane % 32, p);
        }
    };
    auto multiply = [&](uint32_t h, auto products) {
#pragma unroll
        for (uint32_t p = 4 - products.value; p < 4; p++)  // lo lo', lo hi', hi lo', hi hi'
#pragma unroll
            for (uint32_t i = 0; i < WI; i++)
#pragma unroll
                for (uint32_t j = 0; j < WJ; j++)
                    // the right factor's rows first: a lane then holds four consecutive columns of one row
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(r[h][j][p % 2 == 0], l[h][i][p < 2], acc[i][j], 0, 0, 0);
    };
#pragma unroll
    for (uint32_t k = 0; k < NS; k++) fetch(stage(k), k);
    arrived<(NS - 1) * kLoads>();
    read(stage(0), 0);
    auto turn = [&](uint32_t k, uint32_t panel, auto products) {
        constexpr uint32_t kRead = 2 * (WI + WJ), kMfma = decltype(products)::value * WI * WJ, kEach = kMfma > kRead ? kMfma / kRead : 1;
        static_assert(kLoads <= kRead, "");
        read(stage(k), 1);
        multiply(0, products);
#pragma unroll
        for (uint32_t q = 0; q < kRead; q++) {
            __builtin_amdgcn_sched_group_barrier(kSchedMfma, kEach, 0);
            __builtin_amdgcn_sched_group_barrier(kSchedRead, 1, 0);
        }
        // the next stage is there, and all have read this one, which the next loads fill
        __builtin_amdgcn_sched_barrier(0);
        arrived<(NS - 2) * kLoads>();
        __builtin_amdgcn_sched_barrier(0);
        read(stage((k + 1) % NS), 0);
        fetch(stage(k), panel + NS);
        multiply(1, products);
#pragma unroll
        for (uint32_t q = 0; q < kRead; q++) {
            __builtin_amdgcn_sched_group_barrier(kSchedMfma, kEach, 0);
            __builtin_amdgcn_sched_group_barrier(kSchedRead, 1, 0);
            if (q < kLoads) __builtin_amdgcn_sched_group_barrier(kSchedLoad, 1, 0);
        }
    };
    // A matrix instruction cuts its sum off instead of rounding it: of the sums of many positive terms, a bit less each
    // time (at 1433 of them 3e-6 of the result).  Fine results take two turns' sums to a total that is rounded.
    f32x16 total[WI][WJ] = {};
    auto to_total = [&] {
        if constexpr (kFine<OUT>)
#pragma unroll
            for (uint32_t b = 0; b < WI * WJ; b++) {
                total[b / WJ][b % WJ] += acc[b / WJ][b % WJ];
                acc[b / WJ][b % WJ] = f32x16{};
            }
    };
    auto loop = [&](auto products) {
        uint32_t panel = 0;
        for (; panel + NS <= panels; panel += NS)  // whole rounds of the stages, without a way out: the compiler counts the loads
#pragma unroll
            for (uint32_t k = 0; k < NS; k++) {
                turn(k, panel + k, products);
                if (k % 2 == 1) to_total();
            }
#pragma unroll
        for (uint32_t k = 0; k + 1 < NS; k++)
            if (panel + k < panels) turn(k, panel + k, products);
    };
    typedef std::integral_constant<uint32_t, 3> Three;
    typedef std::integral_constant<uint32_t, 4> Four;
    if constexpr (kFine<OUT>) {
        if (d.s <= kFourProducts) loop(Four{});
        else loop(Three{});
    } else {
        loop(Three{});
    }
    arrived<0>();  // no load may arrive in LDS that another workgroup has by then
    if constexpr (kFine<OUT>)
#pragma unroll
        for (uint32_t b = 0; b < WI * WJ; b++) acc[b / WJ][b % WJ] += total[b / WJ][b % WJ];
    if (m.pieces > 1) {  // the sums of the piece, joined by the next launch
        float *to = a.pieces + (uint64_t)wg * (T * T) + wave * (T * T / NW) + lane * 4;
#pragma unroll
        for (uint32_t b = 0; b < WI * WJ; b++)
#pragma unroll
            for (uint32_t g = 0; g < 4; g++)
                *(f32x4 *)(to + (b * 4 + g) * 256) = *((const f32x4 *)&acc[b / WJ][b % WJ] + g);
        return;
    }
    constexpr uint32_t kTurnBytes = 32 * kTurnPitch * 4, kTurns = kStage / kTurnBytes;  // that a stage has room for
    static_assert(kTurns * NS >= NW, "");
    uint32_t *turn_lds = (uint32_t *)(stage(wave / kTurns) + wave % kTurns * kTurnBytes);
#pragma unroll
    for (uint32_t b = 0; b < WI * WJ; b++) {
        const uint32_t i = i0 + wi + b / WJ * 32, j = j0 + wj + b % WJ * 32;
        // of a symmetric result the blocks above the diagonal are written as the mirror of those below
        if (i < left_rows && j < right_rows && (kind >= kNsApply || j <= i))
            ns_finish<OUT>(m, d, a, i, j, acc[b / WJ][b % WJ], turn_lds);
    }
}

// A block of 32 x 32 of a product whose summed index was cut: a workgroup adds up its pieces, a quarter of them
// per wave, in an order that only their number decides.  One workgroup per block of each tile.  4.2 us for
// 640 KB of pieces, which is the launch; 0.29 us more per MB.
template <int OUT, typename C, int N>
__global__ __launch_bounds__(256) void ns_join_kernel(NsList<N> t, NsArgs a) {
    constexpr uint32_t T = C::edge, WI = C::wi, WJ = C::wj, kBlocks = T * T / 1024;
    // The table counts items, a work's tiles once for every piece: each lane its works' tiles, and the sums of those before.
    const uint32_t item = blockIdx.x / kBlocks, block = blockIdx.x % kBlocks;
    uint32_t q = 0, before = 0;
    for (uint32_t q0 = 0; q0 < t.n; q0 += 64) {
        const uint32_t at = q0 + (threadIdx.x & 63);
        uint32_t scan = at < t.n ? tile_at(t.w[at], sides(t.w[at].rows, t.w[at].cols), 0, T).tiles : 0;
        for (int off = 1; off < 64; off <<= 1) {
            const uint32_t up = __shfl_up(scan, off, 64);
            if ((threadIdx.x & 63) >= (uint32_t)off) scan += up;
        }
        const uint32_t n = __popcll(__ballot(at < t.n && before + scan <= item));  // works that end before it
        q += n;
        if (n < 64) {
            if (n > 0) before += __builtin_amdgcn_readlane(scan, n - 1);
            break;
        }
        before += __builtin_amdgcn_readlane(scan, 63);
    }
    const uint32_t k = item - before;
    const NsWork &m = t.w[q];
    const Sides d = sides(m.rows, m.cols);
    const Tile tile = tile_at(m, d, k, T);
    const bool full = (m.op & 15) >= kNsApply;
    const uint32_t wave_of = block / (WI * WJ), b = block % (WI * WJ), lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t i = tile.ti * T + wave_of / 2 * (32 * WI) + b / WJ * 32, j = tile.tj * T + wave_of % 2 * (32 * WJ) + b % WJ * 32;
    if (i >= d.S || j >= (full ? d.L : d.S) || (!full && j > i)) return;
    const float *from = a.pieces + (uint64_t)(m.begin + k) * (T * T) + (wave_of * (WI * WJ) + b) * 1024 + lane * 4;
    f32x4 sum[4] = {};
    for (uint32_t p = m.pieces * wave / 4; p < m.pieces * (wave + 1) / 4; p++)
#pragma unroll
        for (uint32_t g = 0; g < 4; g++) sum[g] += *(const f32x4 *)(from + (uint64_t)p * tile.tiles * (T * T) + g * 256);
    __shared__ f32x4 part[3][4][64];
    __shared__ __align__(16) uint32_t turn[32 * kTurnPitch];
    if (wave > 0)
#pragma unroll
        for (uint32_t g = 0; g < 4; g++) part[wave - 1][g][lane] = sum[g];
    __syncthreads();
    if (wave > 0) return;
    f32x16 acc;
#pragma unroll
    for (uint32_t g = 0; g < 4; g++)
        *((f32x4 *)&acc + g) = (sum[g] + part[0][g][lane]) + (part[1][g][lane] + part[2][g][lane]);
    ns_finish<OUT>(m, d, a, i, j, acc, turn);
}

// -------------------------------------------------------- narrow matrices

// Matrices whose shorter side is at most 128 take a launch per step instead of
// three or four: the work of each is too little to be worth the launches (4.5 us each, of which
// 1.3 pass before the kernel's first instruction).  A workgroup owns kNarrowCols * subs columns
// of X.  It adds up the parts of A = X X^T that all workgroups of its matrix left
// at the launch before, forms M in LDS, takes its columns through X <- M X, and leaves
// its part of the next A.  Each workgroup forms M for itself: 128^3 multiply-adds, three times, 1.5 us.
// Bound by the dependent stages of a launch: 6 us a launch at 64 x 64, 12 at 128 x 128, 16 at 128 x 1024.
//
// LDS, two-plane panels as in memory with the product's swizzle: A and then M
// [s][s], the columns' X^T [64][s], and X [s][64] for the next A.
template <typename F>
__device__ inline void put_block(char *lds, uint32_t rows, uint32_t i0, uint32_t j0, bool mirror, F value) {
    const uint32_t lane = threadIdx.x & 63, i = i0 + lane % 32;
#pragma unroll
    for (uint32_t g = 0; g < 4; g++) {
        const uint32_t j = j0 + 8 * g + 4 * (lane / 32);
        f16x4 hi, lo;
#pragma unroll
        for (int e = 0; e < 4; e++) {
            _Float16 h, w;
            split(value(g, e), h, w);
            hi[e] = h;
            lo[e] = w;
        }
        if (mirror) {  // element (j + e, i)
#pragma unroll
            for (int e = 0; e < 4; e++) {
                char *row = lds + ((i / 32) * rows + j + e) * 128;
                const uint32_t turn = (j + e) / 2 % 8, c = i % 32 / 8, at = i % 8 * 2;
                *(_Float16 *)(row + ((c ^ turn) * 16) + at) = hi[e];
                *(_Float16 *)(row + (((c + 4) ^ turn) * 16) + at) = lo[e];
            }
        } else {
            char *row = lds + ((j / 32) * rows + i) * 128;
            const uint32_t turn = i / 2 % 8, c = j % 32 / 8, at = j % 8 * 2;
            *(f16x4 *)(row + ((c ^ turn) * 16) + at) = hi;
            *(f16x4 *)(row + (((c + 4) ^ turn) * 16) + at) = lo;
        }
    }
}
// Elements (i, j) to (i, j + 3), j a multiple of 4.
__device__ inline void get_entries(const char *lds, uint32_t rows, uint32_t i, uint32_t j, float *v) {
    const char *row = lds + ((j / 32) * rows + i) * 128;
    const uint32_t turn = i / 2 % 8, c = j % 32 / 8, at = j % 8 * 2;
    const f16x4 hi = *(const f16x4 *)(row + ((c ^ turn) * 16) + at), lo = *(const f16x4 *)(row + (((c + 4) ^ turn) * 16) + at);
#pragma unroll
    for (int e = 0; e < 4; e++) v[e] = (float)hi[e] + (float)lo[e];
}
// Rows i0 on of `left` times rows j0 on of `right`, over `panels` panels: hi hi' is added to acc, the rest, before it,
// to small (which may be acc).
template <uint32_t PRODUCTS>
__device__ inline void multiply_blocks(const char *left, uint32_t left_rows, uint32_t i0, const char *right, uint32_t right_rows,
                                       uint32_t j0, uint32_t panels, f32x16 &acc, f32x16 &small) {
    const uint32_t lane = threadIdx.x & 63, i = i0 + lane % 32, j = j0 + lane % 32;
    for (uint32_t p = 0; p < panels; p += 2) {  // a multiple of two: every read of two panels before their products
        f16x8 lh[4], ll[4], rh[4], rl[4];
#pragma unroll
        for (uint32_t h = 0; h < 4; h++) {
            const char *l = left + ((p + h / 2) * left_rows + i) * 128, *r = right + ((p + h / 2) * right_rows + j) * 128;
            const uint32_t c = h % 2 * 2 + lane / 32;
            lh[h] = *(const f16x8 *)(l + ((c ^ (i / 2 % 8)) * 16));
            rl[h] = *(const f16x8 *)(r + (((c + 4) ^ (j / 2 % 8)) * 16));
            ll[h] = *(const f16x8 *)(l + (((c + 4) ^ (i / 2 % 8)) * 16));
            rh[h] = *(const f16x8 *)(r + ((c ^ (j / 2 % 8)) * 16));
        }
#pragma unroll
        for (uint32_t h = 0; h < 4; h++) {
            if constexpr (PRODUCTS == 4) small = __builtin_amdgcn_mfma_f32_32x32x16_f16(rl[h], ll[h], small, 0, 0, 0);
            small = __builtin_amdgcn_mfma_f32_32x32x16_f16(rl[h], lh[h], small, 0, 0, 0);
            small = __builtin_amdgcn_mfma_f32_32x32x16_f16(rh[h], ll[h], small, 0, 0, 0);
        }
#pragma unroll
        for (uint32_t h = 0; h < 4; h++) acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(rh[h], lh[h], acc, 0, 0, 0);
    }
}

// first: X is X0, and only its A is formed.  Parts are read from `from` and left in `to`.
template <int OUT, int N>
__global__ __launch_bounds__(512) void ns_narrow_kernel(NsList<N> t, NsArgs a, const float *from, float *to, uint32_t part_floats,
                                                        int first, int last) {
    const NsWork &m = t.w[find(t.w, t.n, blockIdx.x)];
    const Sides d = sides(m.rows, m.cols);
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t S = d.S, nb = S / 32, lower = nb * (nb + 1) / 2, wg = blockIdx.x - m.begin;
    const uint32_t subs = m.op >> 20, groups = m.pieces;
    extern __shared__ __align__(1024) char lds[];
    char *sq = lds, *xt = lds + S * S * 4, *xg = xt + kNarrowCols * S * 4;
    const float *parts = from + (uint64_t)m.begin * part_floats;
    float *part = to + (uint64_t)blockIdx.x * part_floats;
    // the blocks of A that this wave looks after: `wave` and `wave` + 8 of the lower triangle, row by row
    auto block_of = [&](uint32_t b, uint32_t &bi, uint32_t &bj) {
        bi = b < 1 ? 0 : b < 3 ? 1 : b < 6 ? 2 : 3;
        bj = b - bi * (bi + 1) / 2;
    };
    // 16-byte pieces of X^T's rows (for X0: of X's columns), of a turn's 64 columns, loaded a turn ahead
    char *const mem = buffer(a, m.base, d, first ? 0 : 1);
    const uint32_t rows = first ? S : kNarrowCols, panels = first ? kNarrowCols / 32 : nb, in_turn = panels * rows * 8;
    auto piece_at = [&](uint32_t k, uint32_t l0) {  // of piece k: its place in memory
        const uint32_t p = k / (rows * 8), r = k / 8 % rows;
        return mem + (first ? ((uint64_t)(l0 / 32 + p) * S + r) : ((uint64_t)p * d.L + l0 + r)) * 128 + k % 8 * 16;
    };
    auto swizzled = [&](uint32_t k) { return k / 8 * 128 + ((k % 8) ^ (k / 8 % rows / 2 % 8)) * 16; };
    constexpr uint32_t kPieces = kNarrowShort / 32 * kNarrowCols * 8 / 512;  // of a thread, at most
    u32x4 ahead[kPieces] = {};
    auto fetch = [&](uint32_t sub) {
        const uint32_t l0 = (wg * subs + sub) * kNarrowCols;
        if (sub >= subs || l0 >= d.L) return;
#pragma unroll
        for (uint32_t q = 0; q < kPieces; q++)
            if (threadIdx.x + 512 * q < in_turn) ahead[q] = *(const u32x4 *)piece_at(threadIdx.x + 512 * q, l0);
    };
    fetch(0);
    if (!first) {
        f32x16 v[2] = {};
#pragma unroll
        for (uint32_t q = 0; q < 2; q++) {
            const uint32_t b = wave + 8 * q;
            if (b >= lower) continue;
#pragma unroll 8
            for (uint32_t p = 0; p < groups; p++)
#pragma unroll
                for (uint32_t g = 0; g < 4; g++)
                    *((f32x4 *)&v[q] + g) += *(const f32x4 *)(parts + (uint64_t)p * part_floats + b * 1024 + g * 256 + lane * 4);
            uint32_t bi, bj;
            block_of(b, bi, bj);
            auto value = [&](uint32_t g, int e) { return v[q][4 * g + e] * (kAScale / (kXScale * kXScale)); };
            put_block(sq, S, bi * 32, bj * 32, false, value);
            if (bi != bj) put_block(sq, S, bi * 32, bj * 32, true, value);
        }
        __syncthreads();
#pragma unroll
        for (uint32_t q = 0; q < 2; q++) {
            const uint32_t b = wave + 8 * q;
            if (b >= lower) continue;
            uint32_t bi, bj;
            block_of(b, bi, bj);
            f32x16 acc = {}, small = {};
            multiply_blocks<kFine<OUT> ? 4 : 3>(sq, S, bi * 32, sq, S, bj * 32, nb, acc, small);
#pragma unroll
            for (uint32_t g = 0; g < 4; g++) {
                const uint32_t i = bi * 32 + lane % 32, j = bj * 32 + 8 * g + 4 * (lane / 32);
                float old[4];
                get_entries(sq, S, i, j, old);
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const double square = ((double)acc[4 * g + e] + (double)small[4 * g + e]) * (1.0 / kAScale);
                    v[q][4 * g + e] = polynomial(a, old[e], square, i == j + e);
                }
            }
        }
        __syncthreads();
#pragma unroll
        for (uint32_t q = 0; q < 2; q++) {
            const uint32_t b = wave + 8 * q;
            if (b >= lower) continue;
            uint32_t bi, bj;
            block_of(b, bi, bj);
            auto value = [&](uint32_t g, int e) { return v[q][4 * g + e]; };
            put_block(sq, S, bi * 32, bj * 32, false, value);
            if (bi != bj) put_block(sq, S, bi * 32, bj * 32, true, value);
        }
    }
    f32x16 gram[2] = {};
    for (uint32_t sub = 0; sub < subs; sub++) {
        const uint32_t l0 = (wg * subs + sub) * kNarrowCols;
        if (l0 >= d.L) break;
#pragma unroll
        for (uint32_t q = 0; q < kPieces; q++)
            if (threadIdx.x + 512 * q < in_turn) *(u32x4 *)((first ? xg : xt) + swizzled(threadIdx.x + 512 * q)) = ahead[q];
        fetch(sub + 1);
        __syncthreads();
        if (!first) {
            // blocks (bi, bj) of X' [s][64]: 2 nb of them, one per wave
            const uint32_t bi = wave / 2, bj = wave % 2;
            f32x16 acc = {}, small = {};
            if (bi < nb) multiply_blocks<kFine<OUT> ? 4 : 3>(sq, S, bi * 32, xt, kNarrowCols, bj * 32, nb, acc, small);
            acc += small;
            if (last) {
                if (bi < nb) ns_result<OUT>(m, d, a, bi * 32 + lane % 32, l0 + bj * 32, acc);
                __syncthreads();
                continue;
            }
            __syncthreads();
            if (bi < nb) {
                auto value = [&](uint32_t g, int e) { return acc[4 * g + e] * (1.0f / kAScale); };
                put_block(xg, S, bi * 32, bj * 32, false, value);
                put_block(xt, kNarrowCols, bi * 32, bj * 32, true, value);
            }
            __syncthreads();
            for (uint32_t k = threadIdx.x; k < in_turn; k += 512) *(u32x4 *)piece_at(k, l0) = *(const u32x4 *)(xt + swizzled(k));
        }
#pragma unroll
        for (uint32_t q = 0; q < 2; q++) {
            const uint32_t b = wave + 8 * q;
            if (b >= lower) continue;
            uint32_t bi, bj;
            block_of(b, bi, bj);
            multiply_blocks<kFine<OUT> ? 4 : 3>(xg, S, bi * 32, xg, S, bj * 32, kNarrowCols / 32, gram[q], gram[q]);
        }
        __syncthreads();
    }
    if (last) return;
#pragma unroll
    for (uint32_t q = 0; q < 2; q++) {
        const uint32_t b = wave + 8 * q;
        if (b >= lower) continue;
#pragma unroll
        for (uint32_t g = 0; g < 4; g++) *(f32x4 *)(part + b * 1024 + g * 256 + lane * 4) = *((const f32x4 *)&gram[q] + g);
    }
}

// ---------------------------------------------------------------- launchers

namespace {

// The table in as few arguments as it fits.
template <typename F>
void with_table(const NsTable &t, F launch) {
    if (t.n > (uint32_t)kNsFew) return launch(t);
    NsMats<kNsFew> few;
    std::copy(t.m, t.m + t.n, few.m);
    few.n = t.n;
    few.parts = t.parts;
    launch(few);
}
template <typename F>
void with_table(const NsWorks &t, F launch) {
    if (t.n > (uint32_t)kNsFew) return launch(t);
    NsList<kNsFew> few;
    std::copy(t.w, t.w + t.n, few.w);
    few.n = t.n;
    few.mixed = t.mixed;
    launch(few);
}

template <int N>
void sums(int src, const NsMats<N> &t, const NsArgs &a, uint32_t groups, hipStream_t s) {
    switch (src) {
        case kNsF32: ns_sum_kernel<kNsF32><<<groups, 256, 0, s>>>(t, a); break;
        case kNsFP16: ns_sum_kernel<kNsFP16><<<groups, 256, 0, s>>>(t, a); break;
        case kNsBF16: ns_sum_kernel<kNsBF16><<<groups, 256, 0, s>>>(t, a); break;
        case kNsMuonF32: muon_sum_kernel<kNsMuonF32><<<groups, 256, 0, s>>>(t, a); break;
        case kNsMuonFP16: muon_sum_kernel<kNsMuonFP16><<<groups, 256, 0, s>>>(t, a); break;
        default: muon_sum_kernel<kNsMuonI8><<<groups, 256, 0, s>>>(t, a); break;
    }
}
template <int N>
void prepare(int src, const NsMats<N> &t, const NsArgs &a, uint32_t groups, hipStream_t s) {
    switch (src) {
        case kNsF32: ns_prepare_kernel<kNsF32><<<groups, 256, 0, s>>>(t, a); break;
        case kNsFP16: ns_prepare_kernel<kNsFP16><<<groups, 256, 0, s>>>(t, a); break;
        case kNsBF16: ns_prepare_kernel<kNsBF16><<<groups, 256, 0, s>>>(t, a); break;
        case kNsMuonF32: ns_prepare_kernel<kNsMuonF32><<<groups, 256, 0, s>>>(t, a); break;
        case kNsMuonFP16: ns_prepare_kernel<kNsMuonFP16><<<groups, 256, 0, s>>>(t, a); break;
        default: ns_prepare_kernel<kNsMuonI8><<<groups, 256, 0, s>>>(t, a); break;
    }
}
template <typename C, int N>
void product(int out, const NsList<N> &t, const NsArgs &a, uint32_t items, hipStream_t s) {
    switch (out) {
        case kNsF32: ns_product_kernel<kNsF32, C><<<items, 64 * C::waves, 0, s>>>(t, a); break;
        case kNsFP16: ns_product_kernel<kNsFP16, C><<<items, 64 * C::waves, 0, s>>>(t, a); break;
        case kNsBF16: ns_product_kernel<kNsBF16, C><<<items, 64 * C::waves, 0, s>>>(t, a); break;
        default: ns_product_kernel<kNsMuonF32, C><<<items, 64 * C::waves, 0, s>>>(t, a); break;
    }
}
template <typename C, int N>
void join(int out, const NsList<N> &t, const NsArgs &a, uint32_t tiles, hipStream_t s) {
    const uint32_t groups = tiles * (C::edge * C::edge / 1024);
    switch (out) {
        case kNsF32: ns_join_kernel<kNsF32, C><<<groups, 256, 0, s>>>(t, a); break;
        case kNsFP16: ns_join_kernel<kNsFP16, C><<<groups, 256, 0, s>>>(t, a); break;
        case kNsBF16: ns_join_kernel<kNsBF16, C><<<groups, 256, 0, s>>>(t, a); break;
        default: ns_join_kernel<kNsMuonF32, C><<<groups, 256, 0, s>>>(t, a); break;
    }
}

template <int OUT, int N>
hipError_t narrow(const NsList<N> &t, const NsArgs &a, const float *from, float *to, bool first, bool last, uint32_t groups,
                  uint32_t widest, hipStream_t s) {
    const uint32_t lds = widest * widest * 4 + 2 * kNarrowCols * widest * 4;
    if (lds > 65536) {  // beyond the default of 64 KB; at every launch, since it belongs to the current device
        const hipError_t e = hipFuncSetAttribute((const void *)ns_narrow_kernel<OUT, N>, hipFuncAttributeMaxDynamicSharedMemorySize,
                                                 (int)lds);
        if (e != hipSuccess) return e;
    }
    ns_narrow_kernel<OUT><<<groups, 512, lds, s>>>(t, a, from, to, narrow_part(widest), first, last);
    return hipSuccess;
}

}  // namespace

hipError_t launch_ns_sum(int src, const NsTable &t, const NsArgs &a, uint32_t groups, hipStream_t s) {
    with_table(t, [&](const auto &q) { sums(src, q, a, groups, s); });
    return hipGetLastError();
}

hipError_t launch_ns_prepare(int src, const NsTable &t, const NsArgs &a, uint32_t groups, hipStream_t s) {
    with_table(t, [&](const auto &q) { prepare(src, q, a, groups, s); });
    return hipGetLastError();
}

hipError_t launch_ns_product(int out, uint32_t edge, const NsWorks &t, const NsArgs &a, uint32_t items, hipStream_t s) {
    with_table(t, [&](const auto &q) {
        if (edge == 128) product<Big>(out, q, a, items, s);
        else product<Little>(out, q, a, items, s);
    });
    return hipGetLastError();
}

hipError_t launch_ns_join(int out, uint32_t edge, const NsWorks &t, const NsArgs &a, uint32_t tiles, hipStream_t s) {
    with_table(t, [&](const auto &q) {
        if (edge == 128) join<Big>(out, q, a, tiles, s);
        else join<Little>(out, q, a, tiles, s);
    });
    return hipGetLastError();
}

hipError_t launch_ns_narrow(int out, const NsWorks &t, const NsArgs &a, const float *from, float *to, bool first, bool last,
                            uint32_t groups, uint32_t widest, hipStream_t s) {
    hipError_t e = hipSuccess;
    with_table(t, [&](const auto &q) {
        switch (out) {
            case kNsF32: e = narrow<kNsF32>(q, a, from, to, first, last, groups, widest, s); break;
            case kNsFP16: e = narrow<kNsFP16>(q, a, from, to, first, last, groups, widest, s); break;
            case kNsBF16: e = narrow<kNsBF16>(q, a, from, to, first, last, groups, widest, s); break;
            default: e = narrow<kNsMuonF32>(q, a, from, to, first, last, groups, widest, s); break;
        }
    });
    return e != hipSuccess ? e : hipGetLastError();
}

}  // namespace dedloc
