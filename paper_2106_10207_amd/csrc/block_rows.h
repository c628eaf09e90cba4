// Device code that the kernels of rows share (block.hip, block_forward.h, block_grad.h): vectors of a row, the
// generator of the dropout masks, and the sums of the threads that share a row.
#pragma once

#include "block_internal.h"
#include "ops_internal.h"

#include <type_traits>

namespace dedloc {

constexpr int E = 8;  // columns of a vector: one counter of the generator, 16 bytes of a 16-bit type

// A vector as it lies in memory, so that rows on their way take few registers.
template <typename T>
struct Raw {
    T v[E];
};

// N columns from c on of a row, read past the caches (STREAM) or through them.  RAGGED: where the
// row's end cuts them, the row's last N instead, which align() puts in place once they have arrived; else all are there.
typedef unsigned Word2 __attribute__((ext_vector_type(2), aligned(2)));
typedef unsigned Word4 __attribute__((ext_vector_type(4), aligned(2)));
template <int N, bool STREAM, bool RAGGED, typename T>
__device__ inline void load_part(const T *row, uint32_t c, uint32_t width, T *o) {
    typedef std::conditional_t<N * sizeof(T) == 8, Word2, Word4> Word;
    constexpr int WORDS = N * sizeof(T) / sizeof(Word);
    if (RAGGED && width < N) {
#pragma unroll
        for (int i = 0; i < N; i++) o[i] = row[min((uint32_t)i, width - 1)];
        return;
    }
    if (RAGGED) c = min(c, width - N);
    Word w[WORDS];
#pragma unroll
    for (int i = 0; i < WORDS; i++)
        if constexpr (STREAM)
            w[i] = __builtin_nontemporal_load((const Word *)(row + c) + i);
        else
            w[i] = ((const Word *)(row + c))[i];
    __builtin_memcpy(o, w, sizeof w);
}
// What load_part<N, .., true> took for columns from c on, moved to their places, zeros behind the row's end.
template <int N>
__device__ inline void align(float *o, uint32_t c, uint32_t width) {
    if (c + N <= width) return;
    if (width >= N) {
        const uint32_t s = c - (width - N);
#pragma unroll
        for (uint32_t k = 1; k < N; k *= 2) {
            const bool by = s & k;
#pragma unroll
            for (uint32_t i = 0; i < N; i++) o[i] = by ? (i + k < N ? o[i + k] : 0.0f) : o[i];
        }
    }
#pragma unroll
    for (int i = 0; i < N; i++) o[i] = c + i < width ? o[i] : 0.0f;
}
template <int N, bool STREAM, bool RAGGED, typename T>
__device__ inline void store_part(T *row, uint32_t c, uint32_t width, const float *o) {
    typedef std::conditional_t<N * sizeof(T) == 8, Word2, Word4> Word;
    constexpr int WORDS = N * sizeof(T) / sizeof(Word);
    if (!RAGGED || c + N <= width) {
        T t[N];
        Word w[WORDS];
#pragma unroll
        for (int i = 0; i < N; i++) t[i] = (T)o[i];
        __builtin_memcpy(w, t, sizeof w);
#pragma unroll
        for (int i = 0; i < WORDS; i++)
            if constexpr (STREAM)
                __builtin_nontemporal_store(w[i], (Word *)(row + c) + i);
            else
                ((Word *)(row + c))[i] = w[i];
    } else {
#pragma unroll
        for (int i = 0; i < N; i++)
            if (c + i < width) row[c + i] = (T)o[i];
    }
}
// A use of what is on its way, so that it has arrived here.
template <typename T>
__device__ inline void arrive(Raw<T> &r) {
    uint32_t w[sizeof(r) / 4];
    __builtin_memcpy(w, &r, sizeof w);
#pragma unroll
    for (uint32_t i = 0; i < sizeof(r) / 4; i++) asm volatile("" : "+v"(w[i]));
    __builtin_memcpy(&r, w, sizeof w);
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
// 32 by 32 bit products,
//   (c0, c1, c2, c3) <- (hi(M1 c2) ^ c1 ^ k0, lo(M1 c2), hi(M0 c0) ^ c3 ^ k1, lo(M0 c0)),   k0 += W0, k1 += W1
// A counter (column / 8, row, site, step) gives eight 16-bit numbers, one for each column of a vector.  The products are
// what it costs (a quarter of the rate of an addition).  A thread keeps its columns for many rows, and the row
// enters the first round by c1 alone: of the first three rounds' six products five depend on the column or on
// nothing, and are taken once.  From the second round on, the row (T = 64: the same in the whole wave) enters by one product of the scalar unit.
constexpr uint32_t kM0 = 0xD2511F53u, kM1 = 0xCD9E8D57u, kW0 = 0x9E3779B9u, kW1 = 0xBB67AE85u;

__device__ inline uint32_t hi(uint64_t v) { return (uint32_t)(v >> 32); }
__device__ inline uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) { return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96); }

// What a vector's counters have in common.  After round 2 of row r, with s = M0 * (from_row ^ r):
//   c0, c1 column's alone;  c2 = hi(s) ^ two;  c3 = lo(s)
// and round 3's product of c0 is the column's alone too.
struct Mask {
    uint32_t from_row;     // c0 after round 1, but for the row
    uint32_t two;
    uint32_t c1k0;         // c1 ^ round 3's k0
    uint32_t high_k1, low; // of M0 * c0 in round 3, the high word with k1
    __device__ inline void init(const DropArgs &d, uint32_t step, uint32_t vector) {
        const uint64_t a1 = (uint64_t)vector * kM0, b1 = (uint64_t)d.site * kM1;
        from_row = hi(b1) ^ d.key0;
        const uint32_t c1 = (uint32_t)b1, c2 = hi(a1) ^ step ^ d.key1, c3 = (uint32_t)a1;
        const uint64_t b2 = (uint64_t)c2 * kM1;
        const uint32_t c0 = hi(b2) ^ c1 ^ (d.key0 + kW0);
        two = c3 ^ (d.key1 + kW1);
        c1k0 = (uint32_t)b2 ^ (d.key0 + 2 * kW0);
        const uint64_t a3 = (uint64_t)c0 * kM0;
        high_k1 = hi(a3) ^ (d.key1 + 2 * kW1);
        low = (uint32_t)a3;
    }
    // row: with row0
    __device__ inline void words(const DropArgs &d, uint32_t row, uint32_t *o) const {
        const uint64_t s = (uint64_t)(from_row ^ row) * kM0;
        const uint64_t b3 = (uint64_t)(hi(s) ^ two) * kM1;
        uint32_t c0 = hi(b3) ^ c1k0, c1 = (uint32_t)b3, c2 = high_k1 ^ (uint32_t)s, c3 = low;
        uint32_t k0 = d.key0 + 3 * kW0, k1 = d.key1 + 3 * kW1;
#pragma unroll
        for (int r = 3; r < 10; r++) {
            const uint64_t a = (uint64_t)c0 * kM0, b = (uint64_t)c2 * kM1;
            c0 = xor3(hi(b), c1, k0);
            c1 = (uint32_t)b;
            c2 = xor3(hi(a), c3, k1);
            c3 = (uint32_t)a;
            k0 += kW0;
            k1 += kW1;
        }
        o[0] = c0;
        o[1] = c1;
        o[2] = c2;
        o[3] = c3;
    }
    // x * factor where kept.  What is dropped is zero, whatever it held: an infinity or NaN does not pass.
    // SPLIT: x is the halves of two vectors, the even lane's (the first four columns of both) and the odd lane's
    // (the others); the even lane draws for the first and the odd for the second.
    template <bool SPLIT>
    __device__ inline void apply(const DropArgs &d, uint32_t row, float factor, float *x) const {
        if (d.threshold > 0xffffu) {
#pragma unroll
            for (int i = 0; i < E; i++) x[i] = 0.0f;
            return;
        }
        uint32_t w[4];
        words(d, d.row0 + row, w);
        if (SPLIT) {
            const bool odd = threadIdx.x & 1;
            const uint32_t a = swapped(odd ? w[0] : w[2]), b = swapped(odd ? w[1] : w[3]);
            w[0] = odd ? a : w[0];
            w[1] = odd ? b : w[1];
            w[2] = odd ? w[2] : a;
            w[3] = odd ? w[3] : b;
        }
        select(d, factor, x, w);
    }
    __device__ static inline uint32_t swapped(uint32_t v) {  // with the other of a pair of lanes
        return __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xf, 0xf, true);
    }
    __device__ static inline void select(const DropArgs &d, float factor, float *x, const uint32_t *w) {
        const uint32_t high = d.threshold << 16;  // a word's high half below it: the word below that
#pragma unroll
        for (int i = 0; i < E; i++) {
            const bool gone = i & 1 ? w[i / 2] < high : (uint16_t)w[i / 2] < (uint16_t)d.threshold;
            x[i] = gone ? 0.0f : x[i] * factor;
        }
    }
};

__device__ inline uint32_t step_of(const DropArgs &d) { return d.step + (d.step_at ? (uint32_t)*d.step_at : 0u); }

// --------------------------------------------------------------- sums of a row

template <int CTRL>
__device__ inline float moved(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
// (the lower 32 lanes of a and of b, their upper lanes), and the same of odd and even groups of 16.
struct Pair {
    float x, y;
};
__device__ inline Pair swap32(float a, float b) {
    const auto p = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b), false, false);
    const unsigned x = p[0], y = p[1];  // a bit cast of an element itself takes the first
    return {__builtin_bit_cast(float, x), __builtin_bit_cast(float, y)};
}
__device__ inline Pair swap16(float a, float b) {
    const auto p = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b), false, false);
    const unsigned x = p[0], y = p[1];
    return {__builtin_bit_cast(float, x), __builtin_bit_cast(float, y)};
}

// The sum over aligned groups of T lanes (8 to 64), in all of them.
template <int T>
__device__ inline float lanes_sum(float v) {
    if (T >= 64) {
        const Pair p = swap32(v, v);
        v = p.x + p.y;
    }
    if (T >= 32) {
        const Pair p = swap16(v, v);
        v = p.x + p.y;
    }
    if (T >= 16) v += moved<0x140>(v);  // sixteen, mirrored
    v += moved<0x141>(v);               // eight, mirrored
    v += moved<0x4E>(v);                // the other pair of four
    v += moved<0xB1>(v);                // the other of a pair
    return v;
}
__device__ inline float lane_of(float v, int lane) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane)); }

__device__ inline void barrier() {  // orders LDS alone: rows stay on their way
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// The threads that share a row: T lanes of a wave (T < 64), or `waves` whole waves, then the workgroup
// where there is more than one.  Waves meet in two sets of words in turn: a set is written again only after the barrier
// of the other, which every wave reaches after its reads of the first.  Words of waves that are not there stay zero, so that
// all are read without a count.
template <int MOST>
struct Meet {
    float4 cell[2][MOST / 64];
};

// A thread has V vectors of a row: eight columns in a row, or (SPLIT, rows of fp32) two times four, half a row of threads apart, so that every
// access of a wave is one piece of memory.  RAGGED: the row's end may lie inside such a piece; else a piece is whole or none of it is there.
template <int T, int V, int MOST, bool SPLIT, bool RAGGED>
struct Team {
    static constexpr int PARTS = SPLIT ? 2 : 1, P = E / PARTS;  // pieces of a vector, columns of one
    uint32_t t, lanes, waves, wave, width;
    float inv_width, inv_held, here;
    Meet<MOST> *meet;
    mutable int turn;

    __device__ Team(uint32_t row_waves, uint32_t width_, Meet<MOST> *m) : waves(T < 64 ? 1 : row_waves), width(width_), meet(m), turn(0) {
        lanes = T * waves;
        t = waves > 1 ? threadIdx.x : threadIdx.x & (T - 1);
        wave = T == 64 && waves > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / 64) : 0;
        inv_width = 1.0f / (float)width;
        here = (float)held(wave);
        inv_held = here > 0.0f ? 1.0f / here : 0.0f;
        if (T == 64 && waves > 1) {
            if (threadIdx.x < MOST / 64) meet->cell[0][threadIdx.x] = meet->cell[1][threadIdx.x] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            __syncthreads();
        }
    }
    // the first column of vector v's piece p
    __device__ uint32_t column(int v, int p = 0) const { return SPLIT ? v * lanes * E + (p * lanes + t) * 4 : (v * lanes + t) * E; }
    // the vector of the generator's counters
    __device__ uint32_t counter(int v) const { return SPLIT ? v * lanes + ((t & 1) * lanes + t) / 2 : v * lanes + t; }
    // f(p) for every piece of vector v that is there
    template <typename F>
    __device__ void pieces(int v, F f) const {
#pragma unroll
        for (int p = 0; p < PARTS; p++)
            if (RAGGED || column(v, p) < width) f(p);
    }
    template <bool STREAM, typename D>
    __device__ void load(Raw<D> &r, const D *row, int v, int p) const {
        load_part<P, STREAM, RAGGED>(row, column(v, p), width, r.v + p * P);
    }
    template <bool STREAM, typename D>
    __device__ void store(D *row, int v, int p, const float *o) const {
        store_part<P, STREAM, RAGGED>(row, column(v, p), width, o + p * P);
    }
    template <typename D>
    __device__ void unpack(const Raw<D> &r, int v, float *o) const {
#pragma unroll
        for (int i = 0; i < E; i++) o[i] = (float)r.v[i];
        if constexpr (RAGGED)
#pragma unroll
            for (int p = 0; p < PARTS; p++) align<P>(o + p * P, column(v, p), width);
    }
    // A vector of parameters; `other` where there is none.  Behind the row's end they are zero, and with them what they scale.
    __device__ void parameters(const float *q, int v, float other, float *o) const {
        Raw<float> r = {};
        if (q) {
            pieces(v, [&](int p) { load<false>(r, q, v, p); });
        } else {
            pieces(v, [&](int p) {
#pragma unroll
                for (int i = 0; i < P; i++) r.v[p * P + i] = other;
            });
        }
        unpack(r, v, o);
    }
    // The mean for vector v's column i, zero behind the row's end: x is zero there, and so has to be x - mean, whose product with a
    // large 1 / deviation (equal entries of 2^117 and eps 1e-12: 2^137) no zero of a parameter would make zero again.
    __device__ float about(int v, int i, float mean) const { return column(v, i / P) + (RAGGED ? i % P : 0) < width ? mean : 0.0f; }
    // columns of a row that wave w of it holds
    __device__ uint32_t held(uint32_t w) const {
        uint32_t n = 0;
#pragma unroll
        for (int v = 0; v < V; v++) {
#pragma unroll
            for (int p = 0; p < (SPLIT ? 2 : 1); p++) {
                const uint32_t c = SPLIT ? v * lanes * E + (p * lanes + w * T) * 4 : (v * lanes + w * T) * E;
                n += c >= width ? 0 : min(width - c, (uint32_t)(SPLIT ? T * 4 : T * E));
            }
        }
        return n;
    }
    // Both sums over the lanes that share a row, in a whole wave folded into the halves of one register first: then the first is in the
    // lower lanes of `a`, the second in the upper ones.
    __device__ static void fold2(float &a, float &b) {
        if (T < 64) {
            a = lanes_sum<T>(a);
            b = lanes_sum<T>(b);
        } else {
            const Pair p = swap32(a, b);
            a = lanes_sum<32>(p.x + p.y);
        }
    }
    __device__ static void unfold2(float &a, float &b) {
        if (T < 64) return;
        const Pair p = swap32(a, a);
        a = p.x;
        b = p.y;
    }
    // Both sums in all threads of the row.
    __device__ void sum2(float &a, float &b) const {
        fold2(a, b);
        if (T < 64 || waves == 1) return unfold2(a, b);
        float4 *cell = meet->cell[turn];
        if ((threadIdx.x & 31) == 0) ((float *)(cell + wave))[threadIdx.x >> 5 & 1] = a;
        barrier();
        const float2 mine = *(const float2 *)(cell + (threadIdx.x & (MOST / 64 - 1)));
        a = waves_sum(mine.x);
        b = waves_sum(mine.y);
        turn ^= 1;
    }
    // Every lane holds what the wave of its number left: the sum over the waves.
    __device__ static float waves_sum(float v) {
        if (MOST > 256) return lanes_sum<16>(v);
        v += moved<0x4E>(v);
        return v + moved<0xB1>(v);
    }
    // From a first mean of n terms, the sum of their differences from it and that of the differences' squares: the mean, rounded
    // once, what it lacks, and the squares about the two together.  What the first mean was off by (a rounded sum times
    // a rounded 1 / n) is small whole steps of it, so where all terms are equal nothing here is rounded and m2 becomes zero.
    __device__ static void centre(float n, float inv_n, float sum, float &mean, float &rest, float &m2) {
        const float to = fmaf(sum, inv_n, mean), by = to - mean;
        const float left = fmaf(-n, by, sum);  // the sum of differences from `to`
        m2 = fmaf(-by, sum + left, m2);
        rest = left * inv_n;
        m2 = fmaf(-rest, left, m2);
        m2 = m2 < 0.0f ? 0.0f : m2;  // NaN stays
        mean = to;
    }
    // (mean, sum of squares about it) from the waves' own: no subtraction of large squares.  D: the type that the entries have been
    // rounded to.  The mean of equal entries has to be that entry, or what it is off by stands beside eps as their variance.
    // 16 bits: a wave's sum of equal entries is exact (11 bits, at most 1024 of them) and a quotient put right by its remainder is the entry;
    // of other rows the sum is off by less than the steps between such entries.  fp32: put right by the sum of the differences.
    template <typename D>
    __device__ void moments(const float *x, float &mean, float &m2) const {
        float s = 0.0f, sum = 0.0f, rest = 0.0f;
#pragma unroll
        for (int i = 0; i < V * E; i++) s += x[i];
        s = lanes_sum<T>(s);
        mean = s * inv_held;
        if (sizeof(D) == 2) mean = fmaf(fmaf(-here, mean, s), inv_held, mean);
        m2 = 0.0f;
#pragma unroll
        for (int i = 0; i < V * E; i++) {
            const float d = x[i] - about(i / E, i % E, mean);
            if (sizeof(D) == 4) sum += d;
            m2 = fmaf(d, d, m2);
        }
        if (sizeof(D) == 4) {
            fold2(sum, m2);
            unfold2(sum, m2);
            centre(here, inv_held, sum, mean, rest, m2);
        } else {
            m2 = lanes_sum<T>(m2);
        }
        if (T < 64 || waves == 1) return;
        float4 *cell = meet->cell[turn];
        if ((threadIdx.x & 63) == 0) cell[wave] = make_float4(mean, m2, here, rest);
        barrier();
        const float4 mine = cell[threadIdx.x & (MOST / 64 - 1)];
        mean = waves_sum(mine.z * mine.x) * inv_width;
        const float d = mine.x - mean + mine.w;
        sum = waves_sum(mine.z * d);
        m2 = waves_sum(fmaf(mine.z * d, d, mine.y));
        centre((float)width, inv_width, sum, mean, rest, m2);
        turn ^= 1;
    }
    template <typename D>
    __device__ void sums(const float *x, int kind, float &mean, float &m2) const {
        if (kind == kNormLayer) return moments<D>(x, mean, m2);
        mean = m2 = 0.0f;
#pragma unroll
        for (int i = 0; i < V * E; i++) m2 = fmaf(x[i], x[i], m2);  // zeros behind the row's end
        float none = 0.0f;
        if (T < 64 || waves == 1)
            m2 = lanes_sum<T>(m2);
        else
            sum2(m2, none);
    }
    // The statistics of a norm.  Sums of squares that leave fp32 (entries above 1e18) are taken again of x / 2^96: what that makes
    // too small to square is below 2^-50 of the sum.  Every thread of the row sees the same sum, so all take that way or none.
    template <typename D>
    __device__ float2 stats(float *x, const NormArgs &n) const {
        constexpr float kUnit = 0x1p-96f;
        float mean, m2, eps = n.eps, unit = 1.0f;
        sums<D>(x, n.kind, mean, m2);
        if (__builtin_expect(!(m2 < 0x1p120f), 0)) {
            unit = kUnit;
#pragma unroll
            for (int i = 0; i < V * E; i++) x[i] *= kUnit;
            sums<D>(x, n.kind, mean, m2);
            // eps counts in units of 2^192, if at all; of entries that are all equal there is nothing else
            if (m2 == 0.0f)
                unit = 1.0f;
            else
                eps = eps * kUnit * kUnit;
#pragma unroll
            for (int i = 0; i < V * E; i++) x[i] *= 1.0f / kUnit;
            mean *= 1.0f / kUnit;
        }
        // 1 / sqrt(v): the instruction's (off by 2^-23) and a step that takes its error to the second order
        const float v = fmaf(m2, inv_width, eps), r = __builtin_amdgcn_rsqf(v), h = v * r;
        const float e = fmaf(-h, r, 1.0f) + fmaf(-v, r, h) * r;  // 1 - v r^2, the rounding of h put right
        return make_float2(mean, v < __builtin_inff() ? fmaf(0.5f * r, e, r) * unit : v != v ? v : 0.0f);
    }
};

}  // namespace dedloc
