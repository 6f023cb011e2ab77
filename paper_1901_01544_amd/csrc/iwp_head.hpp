// Kernels of the head's losses: which tokens count, the logits' products with what the softmax needs in their epilogue, the
// logits' gradient, and the two products that take it to the hidden states and to the weight.
//
// Logits z = H W^T are held for one piece of the vocabulary at a time.  Forward, every piece leaves per token and group of
// entries the largest logit m and sum exp(z - m); those are merged into L = log sum exp z.  Backward,
//   dz = c1 (softmax(z) - [label]) + c2 (softmax(z / t) - q)
// replaces the logits of a piece that is still there (the last), and is computed with the logits again for a piece that is not.  A
// vocabulary held as one piece takes 6 T V D operations, in many pieces 8 T V D, but no more memory than one piece's logits.
// 8192 tokens x 2048 x 131072 in fp16, in pieces of 16384 (0.5 GB of logits instead of 4.3): 14.8 ms, a quarter of it for the
// logits' second computation.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/iwp_losses.h"
#include "iwp_matrix.hpp"

namespace iwp {

// A row of dz is held relative to its own token's coefficients: divided by 2^e, the power of two at or below |c1| + |c2|, an entry is less
// than 2 in size.  Times 2^14, fp16 has room for entries down to 2^-38 of the coefficients, the halves of binary32 down to 2^-49, and none
// overflows.  dH's rows take 2^e back one by one.  dW sums over the tokens: its product takes hidden states times 2^(e - the largest
// e), a copy of them that is made where the tokens' powers differ.
constexpr int DZ_BITS = 14;
constexpr int32_t NO_EXPONENT = 1 << 20;           // of coefficients that are 0, infinite or NaN: not scaled, and no other token's concern

struct HeadScalars {
    uint32_t count;        // tokens that count
    int32_t most;          // largest exponent of any token's coefficients, without `scale`
    uint32_t alike;        // 1: all tokens have that one
    uint32_t h_max, w_max; // bits of the largest finite |h|, |w| (of binary32 operands; h: also of fp16 ones that are scaled)
};

struct HeadRows {          // the tokens that count, in order
    uint32_t* token;       // which token the row is
    int32_t* row;          // [tokens] the token's row, -1 if it does not count
    int32_t* label;        // its label, or -1
    float* hard;           // weight * hard where there is a label, else 0
    float* soft;           // weight * soft * t^2 where there are teacher's entries, else 0
    int32_t* exponent;     // of the power of two that its dz is relative to, or NO_EXPONENT
    float* z_label;
    float *lse, *lse_t;    // log sum exp of z, of z / t
};

struct Teacher {           // per token
    int32_t* index;        // [tokens, top], -1: left out, or an index that stands before it
    float* q;              // softmax over the entries; an index that occurs several times has the sum
    float* z;              // by row: the head's logit there
    float* entropy;        // sum q log q, entry by entry
    uint8_t* any;          // 1: there are entries, 2: the label is among them
    uint32_t top;
    float t;
    // The entries by where the logits' product will find them: for every 64 rows, sorted into stretches of `width` vocabulary entries.
    uint32_t *start;       // [rows / 64, stretches + 1]
    uint32_t *found;       // [rows / 64, 64 * top]: place in the stretch, row of the 64, entry
    uint32_t width, stretches;
};
constexpr uint32_t STRETCHES = 8192;               // at most: their counts lie in LDS
__device__ __forceinline__ uint32_t found_word(uint32_t place, uint32_t row, uint32_t k) { return place << 16 | row << 10 | k; }
static_assert(IWP_MAX_TOP <= 1u << 10 && IWP_MAX_VOCAB / STRETCHES <= 1u << 16, "found_word");

// ------------------------------------------------------------------ tokens

// Softmax of the teacher's entries of one token at temperature t; a wavefront per token.  An index that occurs again hands its share to
// the first of its kind, for which every entry is compared with every other in LDS: 11 us for 4096 tokens of 64 entries.
__global__ void __launch_bounds__(256) k_head_teacher(const int32_t* __restrict__ index, const float* __restrict__ logit,
                                                      const int32_t* __restrict__ label, uint32_t tokens, uint32_t vocab, Teacher T) {
    __shared__ int32_t at[4][IWP_MAX_TOP];
    __shared__ float qs[4][IWP_MAX_TOP];
    const uint32_t wave = threadIdx.x >> 6, i = blockIdx.x * 4 + wave, lane = threadIdx.x & 63;
    if (i >= tokens) return;
    const size_t base = (size_t)i * T.top;
    float m = -INFINITY;
    bool any = false, nan = false;
    for (uint32_t k = lane; k < T.top; k += 64) {
        const float s = logit[base + k];
        const int32_t j = index[base + k];
        const bool in = (uint32_t)j < vocab && !(s == -INFINITY);
        at[wave][k] = in ? j : -1;
        qs[wave][k] = s;
        if (in) {
            any = true;
            nan |= s != s;
            m = fmaxf(m, s);
        }
    }
    for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    lanes_exchange();
    any = __ballot(any) != 0;
    if (__ballot(nan)) m = NAN;
    float sum = 0.0f;
    for (uint32_t k = lane; k < T.top; k += 64)
        if (at[wave][k] >= 0) sum += expf((qs[wave][k] - m) / T.t);
    for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
    const float log_sum = logf(sum);
    float entropy = 0.0f;
    for (uint32_t k = lane; k < T.top; k += 64) {
        const bool in = at[wave][k] >= 0;
        const float log_q = (qs[wave][k] - m) / T.t - log_sum, q = in ? expf(log_q) : 0.0f;
        qs[wave][k] = q;
        if (in && q != 0.0f) entropy += q * log_q;
    }
    for (int o = 32; o; o >>= 1) entropy += __shfl_xor(entropy, o);
    lanes_exchange();
    const int32_t y = label ? label[i] : -1;
    bool is_label = false;
    for (uint32_t k = lane; k < T.top; k += 64) {
        const int32_t j = at[wave][k];
        float q = 0.0f;
        bool first = j >= 0;
#pragma unroll 8
        for (uint32_t v = 0; v < T.top; ++v)
            if (at[wave][v] == j) {
                q += qs[wave][v];
                first = first && v >= k;
            }
        T.index[base + k] = first ? j : -1;
        T.q[base + k] = first ? q : 0.0f;
        is_label |= first && j == y;
    }
    is_label = __ballot(is_label) != 0;
    if (lane == 0) {
        T.entropy[i] = entropy;
        T.any[i] = any + 2 * is_label;
    }
}

// One workgroup: numbers the tokens that count, in order, and finds the powers of two of their coefficients.  The products then run over
// those tokens alone: what stands in the others' rows is never read, nor computed with.  Bound by its rounds of 1024 tokens, each two
// barriers: 5 us for 1000 tokens, 9 for 4096, 16 for 8192.
__global__ void __launch_bounds__(1024) k_head_rows(const int32_t* __restrict__ label, const float* __restrict__ weight,
                                                    const uint8_t* __restrict__ any, uint32_t tokens, uint32_t vocab, float hard,
                                                    float soft, float t, HeadRows R, float* __restrict__ loss,
                                                    HeadScalars* __restrict__ S) {
    __shared__ uint32_t in_wave[16];
    __shared__ int32_t most_of[16], least_of[16];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t count = 0;
    int32_t most = -NO_EXPONENT, least = NO_EXPONENT;
    for (uint32_t base = 0; base < tokens; base += 1024) {
        const uint32_t i = base + threadIdx.x;
        float ch = 0.0f, cs = 0.0f;
        int32_t y = -1;
        bool in = false;
        if (i < tokens) {
            const float a = weight ? weight[i] : 1.0f;
            if (label && (uint32_t)label[i] < vocab) y = label[i];
            if (y >= 0) ch = a * hard;
            const bool entries = any && any[i];
            if (entries) cs = a * (soft * t * t);
            in = a != 0.0f && ((y >= 0 && hard != 0.0f) || (entries && soft != 0.0f));
        }
        const uint64_t mask = __ballot(in);
        if (lane == 0) in_wave[wave] = __popcll(mask);
        __syncthreads();
        uint32_t before = count, all = 0;
        for (uint32_t v = 0; v < 16; ++v) {
            if (v < wave) before += in_wave[v];
            all += in_wave[v];
        }
        const uint32_t at = before + __popcll(mask & ((1ull << lane) - 1));
        if (in) {
            R.token[at] = i;
            R.label[at] = y;
            R.hard[at] = ch;
            R.soft[at] = cs;
            const float c1 = fabsf(ch), c2 = fabsf(cs) / t;
            int32_t e = NO_EXPONENT;
            if (c1 < INFINITY && c2 < INFINITY && (c1 != 0.0f || c2 != 0.0f)) {
                e = ilogbf(fmaxf(c1, c2));
                if (c1 + c2 >= ldexpf(1.0f, e + 1)) ++e;       // the sum may be infinite: so is 2^128
                most = max(most, e);
                least = min(least, e);
            }
            R.exponent[at] = e;
        } else if (i < tokens) {
            loss[i] = 0.0f;
        }
        if (i < tokens) R.row[i] = in ? (int32_t)at : -1;
        count += all;
        __syncthreads();
    }
    for (int o = 32; o; o >>= 1) {
        most = max(most, __shfl_xor(most, o));
        least = min(least, __shfl_xor(least, o));
    }
    if (lane == 0) most_of[wave] = most, least_of[wave] = least;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int v = 1; v < 16; ++v) most = max(most, most_of[v]), least = min(least, least_of[v]);
        S->count = count;
        S->alike = most <= least;
        S->most = most == -NO_EXPONENT ? 0 : most;
        S->h_max = S->w_max = 0;
    }
}

// Sorts the teacher's entries of 64 rows into stretches of the vocabulary, for the logits' product, whose wavefronts then find theirs
// without a search.  Inside a stretch their order is nobody's concern.  4096 tokens x 2048 x 32768 with 64 entries: 9 us here and
// 12 us more in the product.  A dot product of its own for every entry, a wavefront each, took 409 us; reading the rows' entries
// in the product's epilogue 190, with all of a wavefront's rows on their way at once 135.
__global__ void __launch_bounds__(1024) k_head_sort(HeadRows R, Teacher T, const HeadScalars* __restrict__ S) {
    __shared__ uint32_t n[STRETCHES], in_wave[16];
    const uint32_t count = S->count, row0 = blockIdx.x * 64, thread = threadIdx.x;
    if (row0 >= count) return;
    const uint32_t entries = min(64u, count - row0) * T.top;
    for (uint32_t b = thread; b < T.stretches; b += 1024) n[b] = 0;
    __syncthreads();
    for (uint32_t e = thread; e < entries; e += 1024) {
        const int32_t j = T.index[(size_t)R.token[row0 + e / T.top] * T.top + e % T.top];
        if (j >= 0) atomicAdd(&n[(uint32_t)j / T.width], 1u);
    }
    __syncthreads();
    uint32_t* start = T.start + (size_t)blockIdx.x * (T.stretches + 1);
    uint32_t before = 0;
    for (uint32_t b0 = 0; b0 < T.stretches; b0 += 1024) {
        const uint32_t b = b0 + thread, mine = b < T.stretches ? n[b] : 0;
        uint32_t sum = mine;
        for (uint32_t o = 1; o < 64; o <<= 1) {
            const uint32_t other = __shfl_up(sum, o);
            if ((thread & 63) >= o) sum += other;
        }
        if ((thread & 63) == 63) in_wave[thread >> 6] = sum;
        __syncthreads();
        uint32_t all = 0, ahead = before;
        for (uint32_t v = 0; v < 16; ++v) {
            if (v < thread >> 6) ahead += in_wave[v];
            all += in_wave[v];
        }
        if (b < T.stretches) {
            n[b] = ahead + sum - mine;
            start[b] = ahead + sum - mine;
        }
        before += all;
        __syncthreads();
    }
    if (thread == 0) start[T.stretches] = before;
    for (uint32_t e = thread; e < entries; e += 1024) {
        const uint32_t row = e / T.top, k = e % T.top;
        const int32_t j = T.index[(size_t)R.token[row0 + row] * T.top + k];
        if (j < 0) continue;
        const uint32_t stretch = (uint32_t)j / T.width, at = atomicAdd(&n[stretch], 1u);
        T.found[(size_t)row0 * T.top + at] = found_word((uint32_t)j - stretch * T.width, row, k);
    }
}

// ------------------------------------------------------------------ operands

// Binary32 operands: x s = hi + 2^-11 lo with hi, lo in fp16 and s the power of two that takes the largest finite |x| to 2^13 or
// just above.  22 bits of an element are kept, fewer where it is below 2^-27 of the largest one.
__device__ __forceinline__ float split_scale(uint32_t max_bits) {
    const int e = max(1, (int)(max_bits >> 23)) - 127;
    return __uint_as_float((uint32_t)min(127 + 13 - e, 254) << 23);
}
// A sum of products of two split operands -> the sum itself.  In two factors, each a power of two that binary32 has: their product may lie
// outside it.
__device__ __forceinline__ float unsplit(float sum, float sp, float sq) { return sum * (1.0f / sp) * (1.0f / sq); }

struct HeadMatrix {        // rows of a caller's matrix; those of `token` alone where it is given, `count` of them
    const void* x;
    int64_t ld;
    uint32_t rows, dim;
    const uint32_t* token;
    const uint32_t* count;
};

// The first `blocks` workgroups take one matrix, the others another; 16 rows of 1024 elements at a time.  Few and large workgroups: each
// ends in an atomic on one word, and those take 20 ns one after the other (75 MB: 19 to 21 us with 320 workgroups, 37 to 41 with
// 2560).  Operands of fp16: one matrix, and only where its rows are about to be scaled (67 MB: 30 us).
template <bool F32>
__global__ void __launch_bounds__(1024) k_head_max(HeadMatrix A, HeadMatrix B, uint32_t blocks, HeadScalars* __restrict__ S) {
    if (!F32 && S->alike) return;
    const bool second = blockIdx.x >= blocks;
    const HeadMatrix M = second ? B : A;
    const uint32_t block = second ? blockIdx.x - blocks : blockIdx.x, n_blocks = second ? gridDim.x - blocks : blocks;
    const uint32_t rows = M.count ? *M.count : M.rows, across = (M.dim + 1023) / 1024, units = (rows + 15) / 16 * across;
    uint32_t m = 0;
    for (uint32_t u = block; u < units; u += n_blocks) {
        const uint32_t r0 = u / across * 16 + threadIdx.x / 256 * 4, c = u % across * 1024 + threadIdx.x % 256 * 4;
        if (c >= M.dim) continue;
        words4 v[4];
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            const uint32_t r = min(r0 + i, rows - 1);
            const int64_t at = (int64_t)(M.token ? M.token[r] : r) * M.ld + c;
            if (!F32) {
                const uint16_t* p = static_cast<const uint16_t*>(M.x) + at;
                halves4_any four = {};
                if (c + 4 <= M.dim) four = *reinterpret_cast<const halves4_any*>(p);
                else for (uint32_t e = 0; c + e < M.dim; ++e) four[e] = p[e];
#pragma unroll
                for (uint32_t e = 0; e < 4; ++e) v[i][e] = __float_as_uint(F16::value(four[e]));
                continue;
            }
            const float* p = static_cast<const float*>(M.x) + at;
            if (c + 4 <= M.dim) {
                v[i] = *reinterpret_cast<const words4*>(p);
            } else {
                v[i] = words4{};
                for (uint32_t e = 0; c + e < M.dim; ++e) v[i][e] = __float_as_uint(p[e]);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t b = v[i][e] & 0x7fffffffu;
                m = max(m, b < 0x7f800000u ? b : 0u);
            }
    }
    for (int o = 32; o; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o));
    __shared__ uint32_t of[16];
    if ((threadIdx.x & 63) == 0) of[threadIdx.x >> 6] = m;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int v = 1; v < 16; ++v) m = max(m, of[v]);
        if (m) atomicMax(second ? &S->w_max : &S->h_max, m);
    }
}

__device__ __forceinline__ void split_f32(float x, float s, uint16_t* hi, uint16_t* lo) {
    const float y = x * s;
    const _Float16 h = (_Float16)y;
    *hi = __builtin_bit_cast(uint16_t, h);
    *lo = __builtin_bit_cast(uint16_t, (_Float16)((y - (float)h) * 2048.0f));
}

// A matrix into rows of ld_out, zeros past its width; with `count`, zeros in the rows behind it up to the next multiple of 64.  Eight
// elements of four rows a thread: four loads on their way.  32003 rows of 1001 in bf16 (130 MB) 28 us, 4.6 TB/s; with one row a thread
// 48 us.  SCALED: where the tokens' exponents differ, also the rows times 2^(the row's exponent - the largest), in binary32 rounded once:
// in bf16 that is exact; fp16 takes them at the scale of the matrix's largest element, as the halves of binary32 are taken.  8192 x 4096 in
// bf16 41 us instead of 31, in a call of 2.86 ms at 16384 entries.
struct Planes { uint16_t *hi, *lo; };              // lo: of binary32 operands
constexpr uint32_t PACK_ROWS = 4;
template <class E, bool F32, bool SCALED>
__global__ void __launch_bounds__(256) k_head_pack(HeadMatrix M, uint32_t first, Spread spread, const uint32_t* __restrict__ max_bits, 
                                                   Planes out, Planes scaled, const int32_t* __restrict__ exponent, uint32_t ld_out,
                                                   const HeadScalars* __restrict__ S) {
    constexpr bool IS_F16 = !F32 && std::is_same<E, F16>::value;
    const uint32_t rows = M.count ? *M.count : M.rows, end = M.count ? (rows + 63) & ~63u : rows;
    const float s = F32 || (SCALED && IS_F16) ? split_scale(*max_bits) : 1.0f;
    const uint32_t c = spread.unit() * 8, r0 = first + spread.row() * PACK_ROWS;
    if (c >= ld_out) return;
    constexpr int WORDS = F32 ? 2 : 1;
    words4 v[PACK_ROWS][WORDS];
#pragma unroll
    for (uint32_t i = 0; i < PACK_ROWS; ++i) {
        const uint32_t r = r0 + i;
#pragma unroll
        for (int w = 0; w < WORDS; ++w) v[i][w] = words4{};
        if (r >= rows) continue;
        const char* p = static_cast<const char*>(M.x) + ((int64_t)(M.token ? M.token[r] : r) * M.ld + c) * (F32 ? 4 : 2);
        if (c + 8 <= M.dim) {
#pragma unroll
            for (int w = 0; w < WORDS; ++w)
                v[i][w] = F32 ? *reinterpret_cast<const words4*>(p + 16 * w) : (words4)*reinterpret_cast<const words4_any*>(p);
        } else {
#pragma unroll
            for (uint32_t e = 0; e < 8; ++e)
                if (c + e < M.dim) {
                    if (F32) v[i][e / 4 % WORDS][e % 4] = reinterpret_cast<const uint32_t*>(p)[e];
                    else v[i][0][e / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[e] << (e % 2 * 16);
                }
        }
    }
    const bool alike = !SCALED || S->alike;
#pragma unroll
    for (uint32_t i = 0; i < PACK_ROWS; ++i) {
        if (r0 + i >= end) break;
        const size_t at = (size_t)(r0 + i) * ld_out + c;
        auto put = [&](const Planes& to, int shift) {
            uint16_t a[8], b[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (F32) {
                    split_f32(ldexpf(__uint_as_float(v[i][e / 4 % WORDS][e % 4]), shift), s, &a[e], &b[e]);
                } else {
                    const uint16_t x = (uint16_t)(v[i][0][e / 2] >> (e % 2 * 16));
                    a[e] = E::bits(ldexpf(E::value(x) * s, shift));
                }
            }
            store8(to.hi + at, a);
            if (F32) store8(to.lo + at, b);
        };
        if (F32) put(out, 0);
        else *reinterpret_cast<words4*>(out.hi + at) = v[i][0];
        if (!alike) {
            const int32_t of = r0 + i < rows ? exponent[r0 + i] : NO_EXPONENT;
            put(scaled, of == NO_EXPONENT ? 0 : of - S->most);
        }
    }
}

// ------------------------------------------------------------------ logits

enum HeadMode { STATISTICS, STATISTICS_KEPT, GRADIENT };

struct HeadPiece {
    uint32_t first, n;      // vocabulary entries of the piece
    uint32_t ld;            // entries per row of `hi` / `lo`, n rounded up to a tile
    uint16_t *hi, *lo;      // logits (while kept) or their gradient, by row
};

struct HeadStats {          // [groups, rows]: a group is the part of the vocabulary that one wavefront of a tile has
    float *m, *sum, *sum_t;
    uint32_t ld;
};

// How the logits of a piece are kept until the statistics are known: binary32, by halves, or for bf16 operands 16 bits of the distance d
// to the group's largest: of the binary32 number 1 + d, which is at least 1, four bits of the exponent and twelve of the
// fraction.  That is off by at most 2^-13 (1 + d), which moves exp(-d) by less than rounding it to bf16 does (2^-8) up to d = 31.  (In
// fp16, d itself would be off by up to 2^-11 d.)  The last code stands for entries without a share: d of more than 65500, or -inf.
constexpr uint32_t ONE = 0x3f800000u, KEPT_SHIFT = 11, KEPT_NONE = 0xffffu;
template <bool WIDE>
__device__ __forceinline__ void keep_logit(float z, float m, uint16_t* hi, uint16_t* lo) {
    if (WIDE) {
        const uint32_t b = __float_as_uint(z);
        *hi = b >> 16;
        *lo = (uint16_t)b;
    } else {
        const uint32_t d = __float_as_uint(m - z + 1.0f) - ONE;
        *hi = (uint16_t)min((d + (1u << (KEPT_SHIFT - 1))) >> KEPT_SHIFT, KEPT_NONE);      // NaN (as of -inf to -inf) is above all numbers
    }
}
template <bool WIDE>
__device__ __forceinline__ float kept_logit(uint16_t hi, uint16_t lo, float m) {
    if (WIDE) return __uint_as_float((uint32_t)hi << 16 | lo);
    return hi == KEPT_NONE ? m - INFINITY : m - (__uint_as_float(ONE + ((uint32_t)hi << KEPT_SHIFT)) - 1.0f);
}

struct RowGradient {        // what a row's dz takes besides its logits
    float c1, c2, lse, lse_t, t_inv;
    __device__ __forceinline__ float softmaxes(float z) const {
        return c1 * exp_of(z - lse) + c2 * exp_of(z * t_inv - lse_t);
    }
};
// Times `scale`, what a product of dz times 2^(DZ_BITS - exponent) is to be multiplied by.
__device__ __forceinline__ float dz_factor(float scale, int32_t exponent) {
    return ldexpf(scale, (exponent == NO_EXPONENT ? 0 : exponent) - DZ_BITS);
}
__device__ __forceinline__ RowGradient row_gradient(const HeadRows& R, uint32_t row, float t, bool soft) {
    RowGradient g;
    const int32_t of = R.exponent[row], by = DZ_BITS - (of == NO_EXPONENT ? 0 : of);
    g.c1 = ldexpf(R.hard[row], by);
    g.c2 = soft ? ldexpf(R.soft[row] / t, by) : 0.0f;
    g.lse = R.lse[row];
    g.lse_t = soft ? R.lse_t[row] : 0.0f;
    g.t_inv = 1.0f / t;
    return g;
}
// dz entry into the planes: one of the operands' type, or the halves of binary32
template <class E, bool F32>
__device__ __forceinline__ void put_dz(float g, uint16_t* hi, uint16_t* lo) {
    if (F32) split_f32(g, 1.0f, hi, lo);
    else *hi = E::bits(g);
}

template <class E, int BP, int BQ, int WP, int WQ, int MODE, bool F32, bool WIDE, bool SOFT>
__global__ void __launch_bounds__(WP * WQ * 64) k_head_logits(Operand W, Operand H, uint32_t dim_padded, HeadPiece G, HeadRows R,
                                                              HeadStats St, Teacher T, const HeadScalars* __restrict__ S) {
    typedef Product<E, BP, BQ, WP, WQ, false, false> M;
    __shared__ __align__(1024) char lds[M::LDS];
    const uint32_t count = S->count;
    uint32_t tp, tq;
    tile_of(blockIdx.x, (G.n + BP - 1) / BP, H.extent / BQ, &tp, &tq);
    if (tq * BQ >= count) return;
    H.extent = count;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t p0 = tp * BP + M::p_of(wave), q0 = tq * BQ + M::q_of(wave);
    // the teacher's entries in this wavefront's stretch of the vocabulary, for the 64 rows that its own are among: the first 64 of them
    // a lane each, from before the product
    constexpr bool PICK = SOFT && MODE != GRADIENT;
    uint32_t found = 0, found_from = 0, found_to = 0;
    const uint32_t* list = nullptr;
    if (PICK && q0 < count) {
        const uint32_t stretch = min((G.first + p0) / T.width, T.stretches - 1);
        const uint32_t* start = T.start + (size_t)(q0 / 64) * (T.stretches + 1) + stretch;
        list = T.found + (size_t)(q0 & ~63u) * T.top;
        found_from = start[0];
        found_to = start[1];
        if (found_from + lane < found_to) found = list[found_from + lane];
    }
    M mm;
    mm.run(W, H, tp * BP, tq * BQ, 0, dim_padded, lds);
    float sw = 1.0f, sh = 1.0f;
    if (F32) sw = split_scale(S->w_max), sh = split_scale(S->h_max);
    const float t = T.t, t_inv = 1.0f / t;
    typedef Rows32<4, BP / WP> Picked;
    static_assert(M::WAVES * Picked::BYTES <= M::LDS, "a wavefront's rows");
    char* picked_lds = lds + wave * Picked::BYTES;
#pragma unroll
    for (int b = 0; b < M::FQ; ++b) {
        const uint32_t q = q0 + b * 32 + (lane & 31);
        const bool row_in = q < count;
        if (F32) {
#pragma unroll
            for (int a = 0; a < M::FP; ++a)
#pragma unroll
                for (int r = 0; r < 16; ++r) mm.acc[a][b][r] = unsplit(mm.acc[a][b][r], sw, sh);
        }
        if (p0 + BP / WP > G.n) {                          // the piece ends in here
#pragma unroll
            for (int a = 0; a < M::FP; ++a)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    mm.acc[a][b][r] = p0 + a * 32 + p_in_fragment(r, lane) < G.n ? mm.acc[a][b][r] : -INFINITY;
        }
        float m = -INFINITY;
        RowGradient g{0.0f, 0.0f, INFINITY, INFINITY, 1.0f};       // of rows that are not there: zeros
        if (MODE != GRADIENT) {
            const int32_t label = row_in ? R.label[q] : -1;
            const uint32_t label_at = label >= 0 ? (uint32_t)label - (G.first + p0) - 4 * (lane >> 5) : ~0u;
            float z_label = 0.0f;
#pragma unroll
            for (int a = 0; a < M::FP; ++a)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    z_label = label_at == a * 32 + p_in_fragment(r, 0) ? mm.acc[a][b][r] : z_label;
                    m = fmaxf(m, mm.acc[a][b][r]);
                }
            // the fragments' 32 entries alternate between the two halves of the wavefront, four at a time
            if (label_at < (uint32_t)(BP / WP) && !(label_at & 4u)) R.z_label[q] = z_label;
            m = fmaxf(m, __shfl_xor(m, 32));
            float sum = 0.0f, sum_t = 0.0f;
            const float from = m == -INFINITY ? 0.0f : m;  // none of the group's entries exist: sums of 0
#pragma unroll
            for (int a = 0; a < M::FP; ++a)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float d = mm.acc[a][b][r] - from;
                    sum += exp_of(d);
                    if (SOFT) sum_t += exp_of(d * t_inv);
                }
            sum += __shfl_xor(sum, 32);
            if (SOFT) sum_t += __shfl_xor(sum_t, 32);
            if (row_in && lane < 32) {
                const size_t at = (size_t)((G.first + p0) / (BP / WP)) * St.ld + q;
                St.m[at] = m;
                St.sum[at] = sum;
                if (SOFT) St.sum_t[at] = sum_t;
            }
        } else if (row_in) {
            g = row_gradient(R, q, t, SOFT);
        }
        if (PICK && found_from < found_to) {               // through LDS, where any lane can take any logit
#pragma unroll
            for (int a = 0; a < M::FP; ++a)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const f32x4 v = {mm.acc[a][b][c * 4], mm.acc[a][b][c * 4 + 1], mm.acc[a][b][c * 4 + 2], mm.acc[a][b][c * 4 + 3]};
                    Picked::put(picked_lds, a * 32 + p_in_fragment(c * 4, lane), lane, &v);
                }
            lanes_exchange();
            const uint32_t stretch = (G.first + p0) / T.width * T.width, rows_from = (q0 & 63u) + b * 32;
            for (uint32_t i = found_from + lane; i < found_to; i += 64) {
                const uint32_t word = i < found_from + 64 ? found : list[i];
                const uint32_t p = (word >> 16) + stretch - (G.first + p0), row = (word >> 10 & 63u) - rows_from;
                if (p < (uint32_t)(BP / WP) && row < 32)
                    T.z[(size_t)(q0 + b * 32 + row) * T.top + (word & 1023u)] = Picked::value(picked_lds, row, p);
            }
            lanes_exchange();
        }
        if (MODE == STATISTICS) continue;
        typedef Rows32<2, BP / WP> Out;
        char* mine = picked_lds;
        constexpr bool TWO = MODE == GRADIENT ? F32 : WIDE;
        uint64_t hi[M::FP][4], lo[M::FP][4];
#pragma unroll
        for (int a = 0; a < M::FP; ++a)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                hi[a][c] = lo[a][c] = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    uint16_t x = 0, y = 0;
                    const float z = mm.acc[a][b][c * 4 + e];
                    if (MODE == GRADIENT) {
                        put_dz<E, F32>(SOFT ? g.softmaxes(z) : g.c1 * exp_of(z - g.lse), &x, &y);
                    } else {
                        keep_logit<WIDE>(z, m, &x, &y);
                    }
                    hi[a][c] |= (uint64_t)x << (16 * e);
                    lo[a][c] |= (uint64_t)y << (16 * e);
                }
            }
#pragma unroll
        for (int plane = 0; plane < (TWO ? 2 : 1); ++plane) {
#pragma unroll
            for (int a = 0; a < M::FP; ++a)
#pragma unroll
                for (int c = 0; c < 4; ++c) Out::put(mine, a * 32 + p_in_fragment(c * 4, lane), lane, plane ? &lo[a][c] : &hi[a][c]);
            uint16_t* to = (plane ? G.lo : G.hi) + (size_t)(q0 + b * 32) * G.ld + p0;
            Out::each(mine, lane, [&](uint32_t row, uint32_t p, quad v) { *reinterpret_cast<quad*>(to + (size_t)row * G.ld + p) = v; });
        }
    }
}

// ------------------------------------------------------------------ statistics and losses

// 16 rows a workgroup, 32 threads a row; groups in a fixed order.  8192 rows x 1024 groups (64 MB): 29 us; with 32 rows a workgroup and 8
// threads a row 70 us, and on 700 rows 18 us against 7, for want of workgroups.
template <bool SOFT>
__global__ void __launch_bounds__(512) k_head_join(HeadStats St, uint32_t groups, HeadRows R, Teacher T, float* __restrict__ loss,
                                                   const HeadScalars* __restrict__ S) {
    constexpr uint32_t ROWS = 16, PARTS = 32;
    __shared__ float ms[PARTS][ROWS], ss[PARTS][ROWS], ts[PARTS][ROWS];
    const uint32_t in = threadIdx.x % ROWS, part = threadIdx.x / ROWS, row = blockIdx.x * ROWS + in, count = S->count;
    if (blockIdx.x * ROWS >= count) return;
    const float t_inv = SOFT ? 1.0f / T.t : 1.0f;
    float m = -INFINITY, s = 0.0f, st = 0.0f, picked = 0.0f;
    auto merge = [&](float m2, float s2, float t2) {
        const float top = fmaxf(m, m2);
        const float a = m == top ? 1.0f : exp_of(m - top), b = m2 == top ? 1.0f : exp_of(m2 - top);
        s = s * a + s2 * b;
        if (SOFT) st = st * (m == top ? 1.0f : exp_of((m - top) * t_inv)) + t2 * (m2 == top ? 1.0f : exp_of((m2 - top) * t_inv));
        m = top;
    };
    if (row < count) {
        constexpr uint32_t AT_ONCE = 4;
        for (uint32_t g0 = part; g0 < groups; g0 += PARTS * AT_ONCE) {
            float gm[AT_ONCE], gs[AT_ONCE], gt[AT_ONCE];
#pragma unroll
            for (uint32_t v = 0; v < AT_ONCE; ++v) {
                const uint32_t g = g0 + v * PARTS;
                const size_t at = (size_t)min(g, groups - 1) * St.ld + row;
                gm[v] = St.m[at];
                gs[v] = St.sum[at];
                gt[v] = SOFT ? St.sum_t[at] : 0.0f;
            }
#pragma unroll
            for (uint32_t v = 0; v < AT_ONCE; ++v)
                if (g0 + v * PARTS < groups) merge(gm[v], gs[v], gt[v]);
        }
        if (SOFT && R.soft[row] != 0.0f) {
            const size_t from = (size_t)R.token[row] * T.top, z = (size_t)row * T.top;
            for (uint32_t k = part; k < T.top; k += PARTS)
                if (T.index[from + k] >= 0) picked += T.q[from + k] * T.z[z + k];
        }
    }
    ms[part][in] = m;
    ss[part][in] = s;
    ts[part][in] = st;
    __syncthreads();
    if (part == 0)
        for (uint32_t v = 1; v < PARTS; ++v) merge(ms[v][in], ss[v][in], ts[v][in]);
    if (SOFT) {
        __syncthreads();
        ms[part][in] = picked;
        __syncthreads();
    }
    if (part || row >= count) return;
    if (SOFT)
        for (uint32_t v = 1; v < PARTS; ++v) picked += ms[v][in];
    const uint32_t token = R.token[row];
    const float lse = m + logf(s);
    float l = 0.0f;
    R.lse[row] = lse;
    if (R.label[row] >= 0 && R.hard[row] != 0.0f) l += R.hard[row] * (lse - R.z_label[row]);
    if (SOFT) {
        const float lse_t = m * t_inv + logf(st);
        R.lse_t[row] = lse_t;
        if (R.soft[row] != 0.0f) l += R.soft[row] * (T.entropy[token] - picked * t_inv + lse_t);
    }
    loss[token] = l;
}

// ------------------------------------------------------------------ the logits' gradient

// Entry k of a row's targets (the teacher's, then the label): where it lies in the piece, and its dz, in binary32 from its logit.  False
// where it lies elsewhere or another entry stands for it.
template <bool SOFT>
__device__ __forceinline__ bool target_dz(uint32_t k, const HeadPiece& G, uint32_t row, uint32_t token, int32_t label, const RowGradient& g,
                                          const HeadRows& R, const Teacher& T, uint32_t* at, float* dz) {
    const uint32_t top = SOFT ? T.top : 0;
    const size_t entry = (size_t)token * top + k;
    const bool teacher = SOFT && k < top;
    const int32_t j = teacher ? T.index[entry] : label;
    if (j < 0 || (uint32_t)j - G.first >= G.n) return false;
    if (SOFT && !teacher && (T.any[token] & 2)) return false;          // an entry of the teacher's is the label: it stands for both
    const float z = teacher ? T.z[(size_t)row * top + k] : R.z_label[row];
    float d = SOFT ? g.softmaxes(z) : g.c1 * exp_of(z - g.lse);
    if (teacher) d -= g.c2 * T.q[entry];
    if (j == label) d -= g.c1;
    *at = (uint32_t)j - G.first;
    *dz = d;
    return true;
}

// In place on a kept piece: a workgroup takes 4096 entries of a row, twice eight a thread.  The label's entry is put right here, the
// teacher's are by k_head_targets (handed around through LDS in here they cost 65 us at 4096 x 32768, there 9).  Bound by memory:
// 8192 x 131072 entries of 2 bytes 750 us, 5.7 TB/s; with eight entries a thread 850.
constexpr uint32_t DZ_ACROSS = 4096;
template <class E, bool F32, bool WIDE, bool SOFT>
__global__ void __launch_bounds__(256) k_head_dz(HeadPiece G, uint32_t first_row, uint32_t group, HeadStats St, HeadRows R, Teacher T,
                                                 const HeadScalars* __restrict__ S) {
    const uint32_t count = S->count, across = (G.ld + DZ_ACROSS - 1) / DZ_ACROSS, row = first_row + blockIdx.x / across;
    const uint32_t first = blockIdx.x % across * DZ_ACROSS + threadIdx.x * 8;
    if (row >= ((count + 63) & ~63u)) return;
    constexpr int PARTS = DZ_ACROSS / 2048;
    uint16_t hi[PARTS][8] = {}, lo[PARTS][8] = {};
    if (row < count) {
        float m[PARTS] = {};
#pragma unroll
        for (int v = 0; v < PARTS; ++v) {
            const uint32_t p = first + v * 2048;
            const size_t at = (size_t)row * G.ld + p;
            if (p < G.ld) {
                load8(G.hi + at, hi[v]);
                if (WIDE) load8(G.lo + at, lo[v]);
                else m[v] = St.m[(size_t)((G.first + p) / group) * St.ld + row];
            }
        }
        const RowGradient g = row_gradient(R, row, T.t, SOFT);
        const uint32_t label = SOFT ? ~0u : (uint32_t)R.label[row] - G.first;
#pragma unroll
        for (int v = 0; v < PARTS; ++v) {
            const uint32_t p = first + v * 2048;
            float d[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float z = kept_logit<WIDE>(hi[v][e], lo[v][e], m[v]);
                d[e] = SOFT ? g.softmaxes(z) : g.c1 * exp_of(z - g.lse);
                if (p + e >= G.n) d[e] = 0.0f;
            }
            if (!SOFT && label - p < 8 && label < G.n) {
                const float is = g.c1 * exp_of(R.z_label[row] - g.lse) - g.c1;
#pragma unroll
                for (uint32_t e = 0; e < 8; ++e)
                    if (label - p == e) d[e] = is;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) put_dz<E, F32>(d[e], &hi[v][e], &lo[v][e]);
        }
    }
#pragma unroll
    for (int v = 0; v < PARTS; ++v) {
        const uint32_t p = first + v * 2048;
        const size_t at = (size_t)row * G.ld + p;
        if (p < G.ld) {
            store8(G.hi + at, hi[v]);
            if (F32) store8(G.lo + at, lo[v]);
        }
    }
}

// A piece's targets, over the gradient that stands there without them; a wavefront per row.
template <class E, bool F32, bool SOFT>
__global__ void __launch_bounds__(256) k_head_targets(HeadPiece G, HeadRows R, Teacher T, const HeadScalars* __restrict__ S) {
    const uint32_t row = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= S->count) return;
    const RowGradient g = row_gradient(R, row, T.t, SOFT);
    for (uint32_t k = threadIdx.x & 63; k <= (SOFT ? T.top : 0u); k += 64) {
        uint32_t at;
        float d;
        if (!target_dz<SOFT>(k, G, row, R.token[row], R.label[row], g, R, T, &at, &d)) continue;
        uint16_t hi, lo;
        put_dz<E, F32>(d, &hi, &lo);
        G.hi[(size_t)row * G.ld + at] = hi;
        if (F32) G.lo[(size_t)row * G.ld + at] = lo;
    }
}

// ------------------------------------------------------------------ gradients

// dH, partial sums: workgroups of split s take a stretch of the piece's vocabulary.  sums: [splits, rows, ld].  T x D is a small product
// with a long sum: 2048 tokens x 1024 make 32 tiles for 256 compute units, and eight splits fill them.
template <class E, int BP, int BQ, int WP, int WQ>
__global__ void __launch_bounds__(WP * WQ * 64) k_head_dh(Operand W, Operand G, uint32_t splits, uint32_t per_split,
                                                          float* __restrict__ sums, uint32_t rows, uint32_t ld, bool add,
                                                          const HeadScalars* __restrict__ S) {
    typedef Product<E, BP, BQ, WP, WQ, true, false> M;
    __shared__ __align__(1024) char lds[M::LDS];
    const uint32_t count = S->count, np = (W.extent + BP - 1) / BP, nq = G.extent / BQ;
    const uint32_t split = blockIdx.x / (np * nq);
    uint32_t tp, tq;
    tile_of(blockIdx.x - split * np * nq, np, nq, &tp, &tq);
    if (tq * BQ >= count) return;
    G.extent = count;
    M mm;
    const uint32_t k_end = (W.summed + BK - 1) & ~(BK - 1), from = min(split * per_split, k_end), to = min(from + per_split, k_end);
    mm.run(W, G, tp * BP, tq * BQ, from, to, lds);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t p0 = tp * BP + M::p_of(wave), q0 = tq * BQ + M::q_of(wave);
#pragma unroll
    for (int b = 0; b < M::FQ; ++b) {
        const uint32_t q = q0 + b * 32 + (lane & 31);
        if (q >= count) continue;
#pragma unroll
        for (int a = 0; a < M::FP; ++a)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const uint32_t p = p0 + a * 32 + p_in_fragment(c * 4, lane);
                if (p >= ld) continue;
                f32x4* to_sum = reinterpret_cast<f32x4*>(sums + ((size_t)split * rows + q) * ld + p);
                f32x4 v = {mm.acc[a][b][c * 4], mm.acc[a][b][c * 4 + 1], mm.acc[a][b][c * 4 + 2], mm.acc[a][b][c * 4 + 3]};
                if (add) v += *to_sum;
                *to_sum = v;
            }
    }
}

// dH: the splits' sums in order, times what dz and W were scaled by, to the token's row; zeros for tokens that do not count.  Four
// entries a thread.
template <int OUT, bool F32>
__global__ void __launch_bounds__(256) k_head_dh_out(const float* __restrict__ sums, uint32_t splits, uint32_t rows, uint32_t ld,
                                                     HeadRows R, uint32_t first, Spread spread, uint32_t tokens, uint32_t dim, float scale, void* __restrict__ dh,
                                                     int64_t ld_dh, const HeadScalars* __restrict__ S) {
    const uint32_t token = first + spread.row(), c = spread.unit() * 4;
    if (token >= tokens || c >= dim) return;
    const int32_t row = R.row[token];
    f32x4 x = {};
    if (row >= 0) {
        const float factor = dz_factor(scale, R.exponent[row]), s = F32 ? 1.0f / split_scale(S->w_max) : 1.0f;
        const float* from = sums + (size_t)row * ld + c;
        const size_t step = (size_t)rows * ld;
        uint32_t v = 0;
        for (; v + 4 <= splits; v += 4) {
            f32x4 y[4];
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) y[i] = *reinterpret_cast<const f32x4*>(from + (v + i) * step);
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) x += y[i];
        }
        for (; v < splits; ++v) x += *reinterpret_cast<const f32x4*>(from + v * step);
        x = x * s * factor;
    }
    const int64_t to = token * ld_dh + c;
    if (c + 4 <= dim && OUT == OUT_F32) {
        *reinterpret_cast<words4*>(static_cast<float*>(dh) + to) = __builtin_bit_cast(words4, x);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c + e < dim) put<OUT>(dh, to + e, x[e]);
    }
}

// dW of a piece: rows of the vocabulary, summed over the rows of tokens.  Where tokens are few it is bound by writing dW: 5 tokens x 768 x
// 8192 7 us, 684 x 1001 x 32003 with rows of odd length 51 to 54 us (90 us while those were written element by element).
template <class E, int BP, int BQ, int WP, int WQ, int OUT, bool F32>
__global__ void __launch_bounds__(WP * WQ * 64) k_head_dw(Operand H, Planes scaled, Operand G, float scale, void* __restrict__ dw, int64_t ld_dw,
                                                          uint32_t first, uint32_t dim, const HeadScalars* __restrict__ S) {
    typedef Product<E, BP, BQ, WP, WQ, true, true> M;
    __shared__ __align__(1024) char lds[M::LDS];
    const uint32_t count = S->count, n = G.extent;
    uint32_t tp, tq;
    tile_of(blockIdx.x, (dim + BP - 1) / BP, (n + BQ - 1) / BQ, &tp, &tq);
    const uint32_t k_end = (count + BK - 1) & ~(BK - 1);
    H.summed = G.summed = k_end;
    const bool alike = S->alike;
    if (!alike) H.hi = scaled.hi, H.lo = F32 ? scaled.lo : nullptr;
    M mm;
    mm.run(H, G, tp * BP, tq * BQ, 0, k_end, lds);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t p0 = tp * BP + M::p_of(wave), q0 = tq * BQ + M::q_of(wave);
    const float factor = dz_factor(scale, S->most);
    const float s = F32 || (std::is_same<E, F16>::value && !alike) ? 1.0f / split_scale(S->h_max) : 1.0f;
    typedef Rows32<OUT == OUT_F32 ? 4 : 2, BP / WP> Out;
    static_assert(M::WAVES * Out::BYTES <= M::LDS, "a wavefront's rows");
    char* mine = lds + wave * Out::BYTES;
    constexpr uint32_t SIZE = OUT == OUT_F32 ? 4 : 2;
#pragma unroll
    for (int b = 0; b < M::FQ; ++b) {
#pragma unroll
        for (int a = 0; a < M::FP; ++a)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                f32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = mm.acc[a][b][c * 4 + e] * s * factor;
                uint64_t four = 0;
                if (OUT != OUT_F32)
#pragma unroll
                    for (int e = 0; e < 4; ++e) four |= (uint64_t)(OUT == OUT_BF16 ? Bf16::bits(v[e]) : F16::bits(v[e])) << (16 * e);
                Out::put(mine, a * 32 + p_in_fragment(c * 4, lane), lane, OUT == OUT_F32 ? (const void*)&v : (const void*)&four);
            }
        Out::each(mine, lane, [&](uint32_t row, uint32_t p, quad v) {
            const uint32_t q = q0 + b * 32 + row;
            if (q >= n || p0 + p >= dim) return;
            char* to = static_cast<char*>(dw) + ((int64_t)(first + q) * ld_dw + p0 + p) * SIZE;
            if (p0 + p + Out::PER_CHUNK <= dim) {
                *reinterpret_cast<words4_any*>(to) = words4_any{v.x, v.y, v.z, v.w};
            } else {
                const uint32_t word[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int e = 0; e < Out::PER_CHUNK; ++e)
                    if (p0 + p + e < dim) {
                        if (OUT == OUT_F32) reinterpret_cast<uint32_t*>(to)[e] = word[e];
                        else reinterpret_cast<uint16_t*>(to)[e] = (uint16_t)(word[e / 2] >> (16 * (e & 1)));
                    }
            }
        });
    }
}

}  // namespace iwp
