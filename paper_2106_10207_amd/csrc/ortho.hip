// gfx950 kernels of the orthogonalised update (Newton-Schulz steps) and the
// Muon step built on it.
//
// With s the shorter side of a matrix and l the longer, X [s][l] is taken
// towards the nearest matrix with orthogonal rows by
//   X0 = G / (|G|_F + eps),   A = X X^T,   B = b A + c A^2,   X <- a X + B X,
// three products a step on the matrix cores.  A singular value far below 1
// grows by a (3.4) in a step, and a rounding error of X with it, so five
// steps multiply it by up to a^5 = 485: operands of 11 bits (fp16) lose 1e-2 of
// the result of an ill-conditioned gradient, 8 bits (bf16) 1e-1.  So every
// operand is held in two fp16 planes, hi + lo, 22 bits, and a product takes
// three of them,
//   hi hi' + hi lo' + lo hi'
// in fp32 accumulators.  X is stored times 2^12, A and B times 2^10: their entries
// are at most about 1.3 and 3, and the low planes of entries of the usual
// size (1 / sqrt(s l)) then stay in fp16's normal range.
//
// Layout of a two-plane matrix: panels of 32 columns, in a panel the rows one after
// the other, 128 bytes each, 64 of hi then 64 of lo.  A turn of a product's loop
// reads a tile's rows of one panel, one piece of memory.  (Row by row, the rows
// of a tile would lie 4 l bytes apart, for most matrices a power of two, and so
// on one of the L2's channels.)
// Both factors of every product have the summed index along their rows (A and
// B are symmetric; X^T is kept beside X).
#include <type_traits>

#include "ops_internal.h"

#ifndef NS_WIDE
#define NS_WIDE 2, 4, 2
#endif
#ifndef NS_SMALL
#define NS_SMALL 1, 1, 4
#endif
namespace dedloc {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

namespace {

constexpr float kXScale = 4096.0f;  // of X
constexpr float kAScale = 1024.0f;  // of A and B

struct Sides {
    uint32_t s, l, S, L;
    bool tall;  // rows > cols: X is the transpose
};
__host__ __device__ inline Sides sides(const NsMat &m) {
    Sides d;
    d.tall = m.rows > m.cols;
    d.s = d.tall ? m.cols : m.rows;
    d.l = d.tall ? m.rows : m.cols;
    d.S = (d.s + kNsPad - 1) / kNsPad * kNsPad;
    d.L = (d.l + kNsPad - 1) / kNsPad * kNsPad;
    return d;
}

// The parts of a matrix' region.
__device__ inline char *at_x(const NsArgs &a, const NsMat &m) { return a.ws + m.base; }
__device__ inline char *at_xt(const NsArgs &a, const NsMat &m, const Sides &d, int k) {
    return a.ws + m.base + (uint64_t)(1 + k) * d.S * d.L * 4;
}
__device__ inline char *at_a(const NsArgs &a, const NsMat &m, const Sides &d) {
    return a.ws + m.base + (uint64_t)3 * d.S * d.L * 4;
}
__device__ inline char *at_b(const NsArgs &a, const NsMat &m, const Sides &d) {
    return at_a(a, m, d) + (uint64_t)d.S * d.S * 4;
}
// Byte offset of element (i, j) of a matrix of `rows` rows: its hi; lo is 64 bytes on.
__device__ inline uint64_t at_planes(uint32_t i, uint32_t j, uint32_t rows) {
    return ((uint64_t)(j / 32) * rows + i) * 128 + (j % 32) * 2;
}

__device__ inline void split(float v, _Float16 &hi, _Float16 &lo) {
    hi = (_Float16)v;
    lo = (_Float16)(v - (float)hi);
}

// The matrix that workgroup `wg` belongs to.
__device__ inline uint32_t find(const NsTable &t, uint32_t wg) {
    uint32_t k = 0;
    while (k + 1 < t.n && t.m[k + 1].begin <= wg) k++;
    return k;
}

// Entry `e` (flat, absolute) of an averaged gradient.
template <int SRC>
__device__ inline float grad_at(const NsArgs &a, uint64_t e) {
    if (SRC == kNsMuonF32) return ((const float *)a.grad)[e];
    if (SRC == kNsMuonFP16) return (float)((const _Float16 *)a.grad)[e];
    return (float)((const int8_t *)a.grad)[e] * a.scales[e >> 10];
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

// Sums of squares in 64 bits, one per block of kNsTile rows and columns.
template <int SRC>
__global__ __launch_bounds__(256) void ns_sum_kernel(NsTable t, NsArgs a) {
    const NsMat &m = t.m[find(t, blockIdx.x)];
    const uint32_t k = blockIdx.x - m.begin, across = (m.cols + kNsTile - 1) / kNsTile;
    const uint32_t r0 = k / across * kNsTile, col = k % across * kNsTile + threadIdx.x % kNsTile;
    double sum = 0.0;
    if (col < m.cols)
        for (uint32_t r = r0 + threadIdx.x / kNsTile; r < r0 + kNsTile && r < m.rows; r += 256 / kNsTile) {
            const double v = entry<SRC>(a, m, r, col);
            sum = fma(v, v, sum);
        }
    sum = block_sum(sum);
    if (threadIdx.x == 0) a.part[m.part + k] = sum;
}

// Muon: m' = fma(mu, m, g), and the sums of squares of the update, one per
// kSumChunk elements.
template <int SRC>
__global__ __launch_bounds__(256) void muon_sum_kernel(NsTable t, NsArgs a) {
    const NsMat &m = t.m[find(t, blockIdx.x)];
    const uint32_t k = blockIdx.x - m.begin;
    const uint64_t n = (uint64_t)m.rows * m.cols, end = (uint64_t)(k + 1) * kSumChunk < n ? (uint64_t)(k + 1) * kSumChunk : n;
    double sum = 0.0;
    for (uint64_t i = (uint64_t)k * kSumChunk + threadIdx.x; i < end; i += 256) {
        const uint64_t e = m.ld_in + i;
        const float g = grad_at<SRC>(a, e), mom = fmaf(a.mu, a.mom[e], g);
        a.mom[e] = mom;
        const double u = a.nesterov ? fmaf(a.mu, mom, g) : mom;
        sum = fma(u, u, sum);
    }
    sum = block_sum(sum);
    if (threadIdx.x == 0) a.part[m.part + k] = sum;
}

// X0 and its transpose in two planes, zeros in the padding: one workgroup per
// block of 64 x 64 of the matrix as it is stored.
template <int SRC>
__global__ __launch_bounds__(256) void ns_prepare_kernel(NsTable t, NsArgs a) {
    const uint32_t q = find(t, blockIdx.x);
    const NsMat &m = t.m[q];
    const Sides d = sides(m);
    double sum = 0.0;
    const uint32_t end = q + 1 < t.n ? t.m[q + 1].part : t.parts;
    for (uint32_t i = m.part + threadIdx.x; i < end; i += 256) sum += a.part[i];
    sum = block_sum(sum);
    const float scale = (float)((double)kXScale / (sqrt(sum) + (double)a.eps));
    __shared__ float tile[64][65];
    const uint32_t k = blockIdx.x - m.begin;
    const uint32_t across = (d.tall ? d.S : d.L) / 64, r0 = k / across * 64, c0 = k % across * 64;
    const uint32_t tc = threadIdx.x % 64;
    for (uint32_t r = threadIdx.x / 64; r < 64; r += 4) {
        float v = 0.0f;
        if (r0 + r < m.rows && c0 + tc < m.cols) v = entry<SRC>(a, m, r0 + r, c0 + tc) * scale;
        tile[r][tc] = v;
    }
    __syncthreads();
    // the block as stored goes to X (wide) or X^T (tall), its transpose to the other
    char *straight = d.tall ? at_xt(a, m, d, 0) : at_x(a, m), *turned = d.tall ? at_x(a, m) : at_xt(a, m, d, 0);
    const uint32_t h_straight = d.tall ? d.L : d.S, h_turned = d.tall ? d.S : d.L;
    for (uint32_t r = threadIdx.x / 64; r < 64; r += 4) {
        _Float16 hi, lo;
        split(tile[r][tc], hi, lo);
        _Float16 *p = (_Float16 *)(straight + at_planes(r0 + r, c0 + tc, h_straight));
        p[0] = hi;
        p[32] = lo;
        split(tile[tc][r], hi, lo);
        p = (_Float16 *)(turned + at_planes(c0 + r, r0 + tc, h_turned));
        p[0] = hi;
        p[32] = lo;
    }
}

// A block's results: row i, columns j0 + 8 g + (0 to 3) are acc[4 g] to
// acc[4 g + 3].  diagonal: the block lies on a symmetric result's diagonal.
template <int PHASE, int OUT>
__device__ inline void ns_finish(const NsMat &m, const Sides &d, const NsArgs &a, uint32_t i, uint32_t j0, bool diagonal,
                                 const f32x16 &acc) {
#pragma unroll
    for (uint32_t g = 0; g < 4; g++) {
        const uint32_t j = j0 + 8 * g;
        float v[4];
        f16x4 hi, lo;
        if (PHASE == kNsGram) {
            for (int e = 0; e < 4; e++) v[e] = acc[4 * g + e] * (kAScale / (kXScale * kXScale));
        } else {
            const char *old = (PHASE == kNsSquare ? at_a(a, m, d) : at_x(a, m)) + at_planes(i, j, d.S);
            hi = *(const f16x4 *)old;
            lo = *(const f16x4 *)(old + 64);
            for (int e = 0; e < 4; e++) {
                const float o = (float)hi[e] + (float)lo[e];
                v[e] = PHASE == kNsSquare ? fmaf(a.b, o, a.c * (acc[4 * g + e] * (1.0f / kAScale)))
                                          : fmaf(a.a, o, acc[4 * g + e] * (1.0f / kAScale));
            }
        }
        if (PHASE == kNsApply && a.last) {
            for (int e = 0; e < 4; e++) {
                if (i >= d.s || j + e >= d.l) continue;
                const uint32_t row = d.tall ? j + e : i, col = d.tall ? i : j + e;
                const float o = v[e] * (1.0f / kXScale);
                if (OUT == kNsMuonF32) {
                    float *x = a.x + m.ld_in + (uint64_t)row * m.cols + col;
                    *x = fmaf(-m.unit, o, ((m.flags & 1) ? a.keep : 1.0f) * *x);
                } else {
                    const uint64_t at = (uint64_t)row * m.ld_out + col;
                    if (OUT == kNsF32) ((float *)m.out)[at] = o;
                    if (OUT == kNsFP16) ((_Float16 *)m.out)[at] = (_Float16)o;
                    if (OUT == kNsBF16) ((__bf16 *)m.out)[at] = (__bf16)o;
                }
            }
            continue;
        }
        for (int e = 0; e < 4; e++) {
            _Float16 h, w;
            split(v[e], h, w);
            hi[e] = h;
            lo[e] = w;
        }
        char *to = (PHASE == kNsGram ? at_a(a, m, d) : PHASE == kNsSquare ? at_b(a, m, d) : at_x(a, m)) +
                   at_planes(i, j, d.S);
        *(f16x4 *)to = hi;
        *(f16x4 *)(to + 64) = lo;
        if (!diagonal) {  // X^T, or the upper triangle
            char *base = PHASE == kNsGram ? at_a(a, m, d) : PHASE == kNsSquare ? at_b(a, m, d) : at_xt(a, m, d, 1 - a.turn);
            for (int e = 0; e < 4; e++) {
                _Float16 *p = (_Float16 *)(base + at_planes(j + e, i, PHASE == kNsApply ? d.L : d.S));
                p[0] = hi[e];
                p[32] = lo[e];
            }
        }
    }
}

#ifndef NS_WIDE
#define NS_WIDE 2, 4, 1
#endif
#ifndef NS_SMALL
#define NS_SMALL 1, 1, 4
#endif
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

// One tile of a product of a step: 64 WI rows and 64 WJ columns, a quarter per
// wave, WI x WJ blocks of 32 x 32.  OUT: the dtype of the result of the last step's
// apply, or kNsMuonF32 for the update of the parameters.
//
// A turn of the loop takes 32 of the summed index, 128 bytes of a row of either
// factor.  They go from memory into one of NS stages of LDS without passing
// registers, NS - 1 turns ahead, and from there into registers half a turn ahead, so that
// the matrix cores find their operands; loads and reads are dealt out between the products.
// 16-byte piece c of row r lies at place c ^ (r / 2 % 8) of its row, so that 16
// lanes of a read, one row each, meet all 64 banks (with r % 8 two rows met in a bank
// and every read took 8 cycles instead of 4); the load writes lanes in order, so
// the lane picks its source piece instead.
template <int PHASE, int OUT, int WI, int WJ, int NS>
__global__ __launch_bounds__(256, 2) void ns_product_kernel(NsTable t, NsArgs a) {
    constexpr uint32_t TI = 64 * WI, TJ = 64 * WJ, R = WJ / WI;
    // workgroups go round the 8 XCDs: give each a contiguous range of tiles
    const uint32_t per = gridDim.x / 8, odd = gridDim.x % 8, xcd = blockIdx.x % 8;
    const uint32_t wg = xcd * per + min(xcd, odd) + blockIdx.x / 8;
    const NsMat &m = t.m[find(t, wg)];
    const Sides d = sides(m);
    uint32_t k = wg - m.begin, ti, tj;
    if (PHASE == kNsApply) {
        // bands of 8 tile rows, column by column: a tile's neighbours in time share its factors
        const uint32_t across = (d.L + TJ - 1) / TJ, down = (d.S + TI - 1) / TI;
        const uint32_t band = k / (8 * across), high = min(8u, down - band * 8);
        k -= band * 8 * across;
        ti = band * 8 + k % high;
        tj = k / high;
    } else {  // the lower triangle of a symmetric result: tile rows R u to R u + R - 1 have u + 1 tiles
        uint32_t u = (uint32_t)((sqrtf(8.0f / R * k + 1.0f) - 1.0f) * 0.5f);
        while (R * (u + 1) * (u + 2) / 2 <= k) u++;
        while (R * u * (u + 1) / 2 > k) u--;
        k -= R * u * (u + 1) / 2;
        ti = R * u + k / (u + 1);
        tj = k % (u + 1);
    }
    const uint32_t K = PHASE == kNsGram ? d.L : d.S;  // the summed index
    const char *left = PHASE == kNsGram ? at_x(a, m) : PHASE == kNsSquare ? at_a(a, m, d) : at_b(a, m, d);
    const char *right = PHASE == kNsApply ? at_xt(a, m, d, a.turn) : left;
    const uint32_t left_rows = d.S, right_rows = PHASE == kNsApply ? d.L : d.S;

    constexpr uint32_t kStage = (TI + TJ) * 128;
    // one array per stage: the compiler then knows which loads a read has to wait for
    __shared__ __align__(1024) char lds0[kStage], lds1[NS > 1 ? kStage : 16], lds2[NS > 2 ? kStage : 16],
        lds3[NS > 3 ? kStage : 16];
    auto stage = [&](uint32_t k) { return k == 0 ? lds0 : k == 1 ? lds1 : k == 2 ? lds2 : lds3; };
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t wi = wave / 2 * (32 * WI), wj = wave % 2 * (32 * WJ);
    // A load of a wave takes 8 rows.  The panels' rows past the matrix' end lie beyond the descriptor's end and read as 0.
    constexpr uint32_t kLoads = 2 * (WI + WJ);
    const uint32_t from = wave * 1024 + (lane / 8) * 128 + ((lane % 8) ^ ((wave % 2) * 4 + lane / 16)) * 16;
    const uint64_t left_panel = (uint64_t)left_rows * 128, right_panel = (uint64_t)right_rows * 128;
    const uint32_t left_end = (left_rows - ti * TI) * 128, right_end = (right_rows - tj * TJ) * 128;
    left += (uint64_t)ti * TI * 128;
    right += (uint64_t)tj * TJ * 128;
    const uint32_t panels = K / 32;
    auto fetch = [&](char *lds, uint32_t panel) {
        const uint64_t p = min(panel, panels - 1);  // past the end the last once more: the loop then counts its loads
        const auto lrows = __builtin_amdgcn_make_buffer_rsrc((void *)(left + p * left_panel), 0, left_end, kRawBuffer);
        const auto rrows = __builtin_amdgcn_make_buffer_rsrc((void *)(right + p * right_panel), 0, right_end, kRawBuffer);
#pragma unroll
        for (uint32_t q = 0; q < kLoads; q++)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(q < 2 * WI ? lrows : rrows, (LdsPtr)(lds + (q * 32 + wave * 8) * 128), 16,
                                                     from, (q < 2 * WI ? q : q - 2 * WI) * 4096, 0, 0);
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
            for (uint32_t b = 0; b < WJ; b++) r[h][b][p] = one(TI + wj + b * 32 + lane % 32, p);
        }
    };
    auto multiply = [&](uint32_t h) {
#pragma unroll
        for (uint32_t p = 0; p < 3; p++)  // lo hi', hi lo', hi hi'
#pragma unroll
            for (uint32_t i = 0; i < WI; i++)
#pragma unroll
                for (uint32_t j = 0; j < WJ; j++)
                    // the right factor's rows first: a lane then holds four consecutive columns of one row
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(r[h][j][p == 1], l[h][i][p == 0], acc[i][j], 0, 0, 0);
    };
#pragma unroll
    for (uint32_t k = 0; k < NS; k++) fetch(stage(k), k);
    arrived<(NS - 1) * kLoads>();
    read(stage(0), 0);
    auto turn = [&](uint32_t k, uint32_t panel) {
        read(stage(k), 1);
        multiply(0);
#pragma unroll
        for (uint32_t q = 0; q < kLoads; q++) {
            __builtin_amdgcn_sched_group_barrier(kSchedMfma, 3 * WI * WJ / kLoads, 0);
            __builtin_amdgcn_sched_group_barrier(kSchedRead, 1, 0);
        }
        // the next stage is there, and all have read this one, which the next loads fill
        __builtin_amdgcn_sched_barrier(0);
        arrived<(NS - 2) * kLoads>();
        __builtin_amdgcn_sched_barrier(0);
        read(stage((k + 1) % NS), 0);
        fetch(stage(k), panel + NS);
        multiply(1);
#pragma unroll
        for (uint32_t q = 0; q < kLoads; q++) {
            __builtin_amdgcn_sched_group_barrier(kSchedMfma, 3 * WI * WJ / kLoads, 0);
            __builtin_amdgcn_sched_group_barrier(kSchedRead, 1, 0);
            __builtin_amdgcn_sched_group_barrier(kSchedLoad, 1, 0);
        }
    };
    uint32_t panel = 0;
    for (; panel + NS <= panels; panel += NS)  // whole rounds of the stages, without a way out: the compiler counts the loads
#pragma unroll
        for (uint32_t k = 0; k < NS; k++) turn(k, panel + k);
#pragma unroll
    for (uint32_t k = 0; k + 1 < NS; k++)
        if (panel + k < panels) turn(k, panel + k);
    arrived<0>();  // no load may arrive in LDS that another workgroup has by then
#pragma unroll
    for (uint32_t bi = 0; bi < WI; bi++)
#pragma unroll
        for (uint32_t bj = 0; bj < WJ; bj++) {
            const uint32_t i0 = ti * TI + wi + bi * 32, j0 = tj * TJ + wj + bj * 32;
            // of a symmetric result the blocks above the diagonal are written as the mirror of those below
            if (i0 < left_rows && j0 < right_rows && (PHASE == kNsApply || j0 <= i0))
                ns_finish<PHASE, OUT>(m, d, a, i0 + lane % 32, j0 + 4 * (lane / 32), PHASE != kNsApply && i0 == j0, acc[bi][bj]);
        }
}

// ---------------------------------------------------------------- launchers

hipError_t launch_ns_sum(int src, const NsTable &t, const NsArgs &a, uint32_t groups, hipStream_t s) {
    switch (src) {
        case kNsF32: ns_sum_kernel<kNsF32><<<groups, 256, 0, s>>>(t, a); break;
        case kNsFP16: ns_sum_kernel<kNsFP16><<<groups, 256, 0, s>>>(t, a); break;
        case kNsBF16: ns_sum_kernel<kNsBF16><<<groups, 256, 0, s>>>(t, a); break;
        case kNsMuonF32: muon_sum_kernel<kNsMuonF32><<<groups, 256, 0, s>>>(t, a); break;
        case kNsMuonFP16: muon_sum_kernel<kNsMuonFP16><<<groups, 256, 0, s>>>(t, a); break;
        default: muon_sum_kernel<kNsMuonI8><<<groups, 256, 0, s>>>(t, a); break;
    }
    return hipGetLastError();
}

hipError_t launch_ns_prepare(int src, const NsTable &t, const NsArgs &a, uint32_t groups, hipStream_t s) {
    switch (src) {
        case kNsF32: ns_prepare_kernel<kNsF32><<<groups, 256, 0, s>>>(t, a); break;
        case kNsFP16: ns_prepare_kernel<kNsFP16><<<groups, 256, 0, s>>>(t, a); break;
        case kNsBF16: ns_prepare_kernel<kNsBF16><<<groups, 256, 0, s>>>(t, a); break;
        case kNsMuonF32: ns_prepare_kernel<kNsMuonF32><<<groups, 256, 0, s>>>(t, a); break;
        case kNsMuonFP16: ns_prepare_kernel<kNsMuonFP16><<<groups, 256, 0, s>>>(t, a); break;
        default: ns_prepare_kernel<kNsMuonI8><<<groups, 256, 0, s>>>(t, a); break;
    }
    return hipGetLastError();
}

namespace {
template <int WI, int WJ, int NS>
void product(int phase, int out, const NsTable &t, const NsArgs &a, uint32_t groups, hipStream_t s) {
    if (phase == kNsGram) {
        ns_product_kernel<kNsGram, kNsF32, WI, WJ, NS><<<groups, 256, 0, s>>>(t, a);
    } else if (phase == kNsSquare) {
        ns_product_kernel<kNsSquare, kNsF32, WI, WJ, NS><<<groups, 256, 0, s>>>(t, a);
    } else {
        switch (out) {
            case kNsF32: ns_product_kernel<kNsApply, kNsF32, WI, WJ, NS><<<groups, 256, 0, s>>>(t, a); break;
            case kNsFP16: ns_product_kernel<kNsApply, kNsFP16, WI, WJ, NS><<<groups, 256, 0, s>>>(t, a); break;
            case kNsBF16: ns_product_kernel<kNsApply, kNsBF16, WI, WJ, NS><<<groups, 256, 0, s>>>(t, a); break;
            default: ns_product_kernel<kNsApply, kNsMuonF32, WI, WJ, NS><<<groups, 256, 0, s>>>(t, a); break;
        }
    }
}
}  // namespace

// wide: tiles of 128 x 256, else of 64 x 64 (what `groups` and the table count)
hipError_t launch_ns_product(int phase, int out, bool wide, const NsTable &t, const NsArgs &a, uint32_t groups, hipStream_t s) {
    if (wide) product<NS_WIDE>(phase, out, t, a, groups, s);
    else product<NS_SMALL>(phase, out, t, a, groups, s);
    return hipGetLastError();
}

}  // namespace dedloc
