// Kernels of the head's losses: which tokens count, the logits' products with what the softmax needs in their epilogue, the
// logits' gradient, and the two products that take it to the hidden states and to the weight.
//
// Logits z = H W^T are held for one piece of the vocabulary at a time.  Forward, every piece leaves per token and group of
// entries the largest logit m and sum exp(z - m); those are merged into L = log sum exp z.  Backward,
//   dz = c1 (softmax(z) - [label]) + c2 (softmax(z / t) - q)
// replaces the logits of a piece that is still there, and is computed with the logits again for a piece that is not.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/iwp_losses.h"
#include "iwp_matrix.hpp"

namespace iwp {

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.693147180559945309417f;
// The gradient's coefficients are divided by the largest of any token, so an entry of dz is at most 1 in size.  Times 2^14, fp16
// has room for entries down to 2^-38 of that, and none overflows; bf16 and the halves of binary32 do not mind.
constexpr float DZ_SCALE = 16384.0f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * LOG2E); }

struct HeadScalars {
    uint32_t count;        // tokens that count
    float most;            // largest |c1| + |c2| of any token, without `scale`
    uint32_t h_max, w_max; // bits of the largest finite |h|, |w| (binary32 operands only)
};

struct HeadRows {          // the tokens that count, in order
    uint32_t* token;       // which token the row is
    int32_t* row;          // [tokens] the token's row, -1 if it does not count
    int32_t* label;        // its label, or -1
    float* hard;           // weight * hard where there is a label, else 0
    float* soft;           // weight * soft * t^2 where there are teacher's entries, else 0
    float* z_label;
    float *lse, *lse_t;    // log sum exp of z, of z / t
};

struct Teacher {           // per token
    int32_t* index;        // [tokens, top], -1: left out
    float* q;
    float* z;              // by row: the head's logit there
    float* entropy;        // sum q log q
    uint8_t* any;
    uint32_t top;
    float t;
};

// ------------------------------------------------------------------ tokens

// softmax of the teacher's entries of one token at temperature t; a wavefront per token
__global__ void __launch_bounds__(256) k_head_teacher(const int32_t* __restrict__ index, const float* __restrict__ logit,
                                                      uint32_t tokens, uint32_t vocab, Teacher T) {
    const uint32_t i = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (i >= tokens) return;
    const size_t base = (size_t)i * T.top;
    float m = -INFINITY;
    bool any = false, nan = false;
    for (uint32_t k = lane; k < T.top; k += 64) {
        const float s = logit[base + k];
        if ((uint32_t)index[base + k] < vocab && !(s == -INFINITY)) {
            any = true;
            nan |= s != s;
            m = fmaxf(m, s);
        }
    }
    for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    any = __ballot(any) != 0;
    if (__ballot(nan)) m = NAN;
    float sum = 0.0f;
    for (uint32_t k = lane; k < T.top; k += 64) {
        const float s = logit[base + k];
        if ((uint32_t)index[base + k] < vocab && !(s == -INFINITY)) sum += expf((s - m) / T.t);
    }
    for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
    const float log_sum = logf(sum);
    float entropy = 0.0f;
    for (uint32_t k = lane; k < T.top; k += 64) {
        const float s = logit[base + k];
        const bool in = (uint32_t)index[base + k] < vocab && !(s == -INFINITY);
        const float log_q = (s - m) / T.t - log_sum, q = in ? expf(log_q) : 0.0f;
        T.index[base + k] = in ? index[base + k] : -1;
        T.q[base + k] = q;
        if (in && q != 0.0f) entropy += q * log_q;
    }
    for (int o = 32; o; o >>= 1) entropy += __shfl_xor(entropy, o);
    if (lane == 0) {
        T.entropy[i] = entropy;
        T.any[i] = any;
    }
}

// One workgroup: numbers the tokens that count, in order, and finds the largest coefficient.
__global__ void __launch_bounds__(1024) k_head_rows(const int32_t* __restrict__ label, const float* __restrict__ weight,
                                                    const uint8_t* __restrict__ any, uint32_t tokens, uint32_t vocab, float hard,
                                                    float soft, float t, HeadRows R, float* __restrict__ loss,
                                                    HeadScalars* __restrict__ S) {
    __shared__ uint32_t in_wave[16];
    __shared__ float most_of[16];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t count = 0;
    float most = 0.0f;
    for (uint32_t base = 0; base < tokens; base += 1024) {
        const uint32_t i = base + threadIdx.x;
        float ch = 0.0f, cs = 0.0f;
        int32_t y = -1;
        bool in = false;
        if (i < tokens) {
            const float a = weight ? weight[i] : 1.0f;
            if (label && (uint32_t)label[i] < vocab) y = label[i];
            if (y >= 0) ch = a * hard;
            if (any && any[i]) cs = a * (soft * t * t);
            in = a != 0.0f && ((y >= 0 && hard != 0.0f) || (any && any[i] && soft != 0.0f));
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
            most = fmaxf(most, fabsf(ch) + fabsf(cs) / t);
        } else if (i < tokens) {
            loss[i] = 0.0f;
        }
        if (i < tokens) R.row[i] = in ? (int32_t)at : -1;
        count += all;
        __syncthreads();
    }
    for (int o = 32; o; o >>= 1) most = fmaxf(most, __shfl_xor(most, o));
    if (lane == 0) most_of[wave] = most;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int v = 1; v < 16; ++v) most = fmaxf(most, most_of[v]);
        S->count = count;
        S->most = most;
        S->h_max = S->w_max = 0;
    }
}

// ------------------------------------------------------------------ operands

// Binary32 operands: x s = hi + 2^-11 lo with hi, lo in fp16 and s the power of two that takes the largest finite |x| to 2^13 or
// just above.  22 bits of an element are kept, fewer where it is below 2^-27 of the largest one.
__device__ __forceinline__ float split_scale(uint32_t max_bits) {
    const int e = max(1, (int)(max_bits >> 23)) - 127;
    return __uint_as_float((uint32_t)min(127 + 13 - e, 254) << 23);
}
// A sum of products of two split operands -> the sum itself, in two factors that are normal numbers.
__device__ __forceinline__ float unsplit(float sum, float sp, float sq) { return sum * (1.0f / sp) * (1.0f / sq); }

__global__ void __launch_bounds__(256) k_head_max(const float* __restrict__ x, int64_t ld, uint32_t rows, uint32_t dim,
                                                  const uint32_t* __restrict__ token, const uint32_t* __restrict__ count,
                                                  uint32_t* __restrict__ max_bits) {
    if (count) rows = *count;
    uint32_t m = 0;
    for (uint32_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const float* p = x + (int64_t)(token ? token[r] : r) * ld;
        for (uint32_t c = threadIdx.x; c < dim; c += 256) {
            const uint32_t b = __float_as_uint(p[c]) & 0x7fffffffu;
            if (b < 0x7f800000u) m = max(m, b);
        }
    }
    for (int o = 32; o; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o));
    __shared__ uint32_t of[4];
    if ((threadIdx.x & 63) == 0) of[threadIdx.x >> 6] = m;
    __syncthreads();
    if (threadIdx.x == 0) {
        m = max(max(of[0], of[1]), max(of[2], of[3]));
        if (m) atomicMax(max_bits, m);
    }
}

__device__ __forceinline__ void split_f32(float x, float s, uint16_t* hi, uint16_t* lo) {
    const float y = x * s;
    const _Float16 h = (_Float16)y;
    *hi = __builtin_bit_cast(uint16_t, h);
    *lo = __builtin_bit_cast(uint16_t, (_Float16)((y - (float)h) * 2048.0f));
}

// Rows of a matrix (those of `token` if given, zeros up to the next multiple of 64 behind them) into rows of ld_out, zeros past dim.
template <bool F32>
__global__ void __launch_bounds__(256) k_head_pack(const void* __restrict__ x, int64_t ld, uint32_t rows, uint32_t dim,
                                                   const uint32_t* __restrict__ token, const uint32_t* __restrict__ count,
                                                   const uint32_t* __restrict__ max_bits, uint16_t* __restrict__ hi,
                                                   uint16_t* __restrict__ lo, uint32_t ld_out) {
    const uint32_t end = count ? (*count + 63) & ~63u : rows;
    if (count) rows = *count;
    const float s = F32 ? split_scale(*max_bits) : 1.0f;
    for (uint32_t r = blockIdx.x; r < end; r += gridDim.x) {
        const int64_t from = r < rows ? (int64_t)(token ? token[r] : r) * ld : 0;
        for (uint32_t c = threadIdx.x; c < ld_out; c += 256) {
            const bool in = r < rows && c < dim;
            const size_t at = (size_t)r * ld_out + c;
            if (F32) {
                uint16_t a, b;
                split_f32(in ? static_cast<const float*>(x)[from + c] : 0.0f, s, &a, &b);
                hi[at] = a;
                lo[at] = b;
            } else {
                hi[at] = in ? static_cast<const uint16_t*>(x)[from + c] : (uint16_t)0;
            }
        }
    }
}

// ------------------------------------------------------------------ the tiles' order

// Workgroups go to the chip's eight dies in turn, and each die has an L2 of its own: each takes a stretch of the tiles in an order
// in which some dozens in a row share few rows and columns (8 of Q by as many of P as run at a time).
__device__ __forceinline__ void tile_of(uint32_t block, uint32_t np, uint32_t nq, uint32_t* p, uint32_t* q) {
    const uint32_t n = np * nq, per = n / 8, more = n % 8, die = block % 8, in = block / 8;
    const uint32_t at = die * per + min(die, more) + in;
    constexpr uint32_t TALL = 8;
    const uint32_t group = at / (np * TALL), first = group * TALL, tall = min(TALL, nq - first), rest = at - group * np * TALL;
    *p = rest / tall;
    *q = first + rest % tall;
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

// How the logits of a piece are kept until the statistics are known: for bf16 operands as fp16 differences to the group's largest
// (an error of 2^-12 of the distance to it, where bf16 would round the gradient to 2^-9), otherwise as binary32, by halves.
template <bool WIDE>
__device__ __forceinline__ void keep_logit(float z, float m, uint16_t* hi, uint16_t* lo) {
    if (WIDE) {
        const uint32_t b = __float_as_uint(z);
        *hi = b >> 16;
        *lo = (uint16_t)b;
    } else {
        *hi = F16::bits(z - m);
    }
}
template <bool WIDE>
__device__ __forceinline__ float kept_logit(uint16_t hi, uint16_t lo, float m) {
    return WIDE ? __uint_as_float((uint32_t)hi << 16 | lo) : F16::value(hi) + m;
}

struct RowGradient {        // what a row's dz takes besides its logits
    float c1, c2, lse, lse_t, t_inv;
    __device__ __forceinline__ float softmaxes(float z) const {
        return c1 * exp_of(z - lse) + c2 * exp_of(z * t_inv - lse_t);
    }
};
__device__ __forceinline__ RowGradient row_gradient(const HeadRows& R, uint32_t row, float most, float t, bool soft) {
    RowGradient g;
    const float to = most > 0.0f ? 1.0f : 0.0f, by = most > 0.0f ? most : 1.0f;
    g.c1 = to * R.hard[row] / by * DZ_SCALE;
    g.c2 = soft ? to * (R.soft[row] / t) / by * DZ_SCALE : 0.0f;
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
                                                              HeadStats St, float t, const HeadScalars* __restrict__ S) {
    typedef Product<E, BP, BQ, WP, WQ, false, false> M;
    __shared__ __align__(1024) char lds[M::LDS];
    const uint32_t count = S->count;
    uint32_t tp, tq;
    tile_of(blockIdx.x, (G.n + BP - 1) / BP, H.extent / BQ, &tp, &tq);
    if (tq * BQ >= count) return;
    H.extent = count;
    M mm;
    mm.run(W, H, tp * BP, tq * BQ, 0, dim_padded, lds);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t p0 = tp * BP + M::p_of(wave), q0 = tq * BQ + M::q_of(wave);
    float sw = 1.0f, sh = 1.0f;
    if (F32) sw = split_scale(S->w_max), sh = split_scale(S->h_max);
    const float t_inv = 1.0f / t;
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
        float m = -INFINITY;
        RowGradient g;
        if (MODE != GRADIENT) {
            const int32_t label = row_in ? R.label[q] : -1;
            const uint32_t label_at = label >= 0 ? (uint32_t)label - (G.first + p0) - 4 * (lane >> 5) : ~0u;
            float z_label = 0.0f;
            if (p0 + BP / WP > G.n) {                      // the piece ends in here
#pragma unroll
                for (int a = 0; a < M::FP; ++a)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        mm.acc[a][b][r] = p0 + a * 32 + p_in_fragment(r, lane) < G.n ? mm.acc[a][b][r] : -INFINITY;
            }
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
            g = row_gradient(R, q, S->most, t, SOFT);
        }
        if (MODE == STATISTICS) continue;
        typedef Rows32<2> Out;
        static_assert(BP / WP == Out::ENTRIES && M::WAVES * Out::BYTES <= M::LDS, "a wavefront's rows");
        char* mine = lds + wave * Out::BYTES;
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
                    const uint32_t p = p0 + a * 32 + p_in_fragment(c * 4 + e, lane);
                    const float z = mm.acc[a][b][c * 4 + e];
                    if (MODE == GRADIENT) {
                        const float d = SOFT ? g.softmaxes(z) : g.c1 * exp_of(z - g.lse);
                        put_dz<E, F32>(row_in && p < G.n ? d : 0.0f, &x, &y);
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
            Out::each(mine, lane, [&](uint32_t row, uint32_t p, uint4 v) { *reinterpret_cast<uint4*>(to + (size_t)row * G.ld + p) = v; });
        }
    }
}

// The head's logits at the teacher's entries: a wavefront per entry.
template <class V>
__device__ __forceinline__ float element(const void* x, int64_t at) { return V::value(static_cast<const uint16_t*>(x)[at]); }
struct F32Element {};
template <>
__device__ __forceinline__ float element<F32Element>(const void* x, int64_t at) { return static_cast<const float*>(x)[at]; }

template <class V>
__global__ void __launch_bounds__(256) k_head_picked(const void* __restrict__ h, int64_t ld_h, const void* __restrict__ w, int64_t ld_w,
                                                     uint32_t dim, HeadRows R, Teacher T, const HeadScalars* __restrict__ S) {
    const uint32_t lane = threadIdx.x & 63, count = S->count;
    for (uint64_t at = (uint64_t)blockIdx.x * 4 + (threadIdx.x >> 6); at < (uint64_t)count * T.top; at += (uint64_t)gridDim.x * 4) {
        const uint32_t row = at / T.top, k = at % T.top, token = R.token[row];
        const int32_t j = T.index[(size_t)token * T.top + k];
        float sum = 0.0f;
        if (j >= 0)
            for (uint32_t c = lane; c < dim; c += 64) sum += element<V>(h, token * ld_h + c) * element<V>(w, j * ld_w + c);
        for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
        if (lane == 0) T.z[at] = sum;
    }
}

// ------------------------------------------------------------------ statistics and losses

// 32 rows a workgroup, 8 threads a row; groups in a fixed order.
template <bool SOFT>
__global__ void __launch_bounds__(256) k_head_join(HeadStats St, uint32_t groups, HeadRows R, Teacher T, float* __restrict__ loss,
                                                   const HeadScalars* __restrict__ S) {
    __shared__ float ms[8][32], ss[8][32], ts[8][32];
    const uint32_t in = threadIdx.x & 31, part = threadIdx.x >> 5, row = blockIdx.x * 32 + in, count = S->count;
    if (blockIdx.x * 32 >= count) return;
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
        for (uint32_t g = part; g < groups; g += 8) {
            const size_t at = (size_t)g * St.ld + row;
            merge(St.m[at], St.sum[at], SOFT ? St.sum_t[at] : 0.0f);
        }
        if (SOFT && R.soft[row] != 0.0f) {
            const size_t from = (size_t)R.token[row] * T.top, z = (size_t)row * T.top;
            for (uint32_t k = part; k < T.top; k += 8)
                if (T.index[from + k] >= 0) picked += T.q[from + k] * T.z[z + k];
        }
    }
    ms[part][in] = m;
    ss[part][in] = s;
    ts[part][in] = st;
    __syncthreads();
    if (part == 0)
        for (int v = 1; v < 8; ++v) merge(ms[v][in], ss[v][in], ts[v][in]);
    if (SOFT) {
        __syncthreads();
        ms[part][in] = picked;
        __syncthreads();
    }
    if (part || row >= count) return;
    if (SOFT)
        for (int v = 1; v < 8; ++v) picked += ms[v][in];
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

// In place on a kept piece; eight entries a thread.
template <class E, bool F32, bool WIDE, bool SOFT>
__global__ void __launch_bounds__(256) k_head_dz(HeadPiece G, uint32_t group, HeadStats St, HeadRows R, float t,
                                                 const HeadScalars* __restrict__ S) {
    const uint32_t count = S->count, across = (G.ld + 2047) / 2048, row = blockIdx.x / across;
    const uint32_t p = (blockIdx.x % across * 256 + threadIdx.x) * 8;
    if (row >= ((count + 63) & ~63u) || p >= G.ld) return;
    const size_t at = (size_t)row * G.ld + p;
    uint16_t hi[8] = {}, lo[8] = {};
    if (row < count) {
        const RowGradient g = row_gradient(R, row, S->most, t, SOFT);
        *reinterpret_cast<uint4*>(hi) = *reinterpret_cast<const uint4*>(G.hi + at);
        if (WIDE) *reinterpret_cast<uint4*>(lo) = *reinterpret_cast<const uint4*>(G.lo + at);
        const float m = St.m[(size_t)((G.first + p) / group) * St.ld + row];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float z = kept_logit<WIDE>(hi[e], lo[e], m);
            float d = 0.0f;
            if (p + e < G.n) d = SOFT ? g.softmaxes(z) : g.c1 * exp_of(z - g.lse);
            put_dz<E, F32>(d, &hi[e], &lo[e]);
        }
    }
    *reinterpret_cast<uint4*>(G.hi + at) = *reinterpret_cast<const uint4*>(hi);
    if (F32) *reinterpret_cast<uint4*>(G.lo + at) = *reinterpret_cast<const uint4*>(lo);
}

// The label's and the teacher's entries of dz, in binary32 from their logits and rounded once.
template <class E, bool F32, bool SOFT>
__global__ void __launch_bounds__(256) k_head_targets(HeadPiece G, HeadRows R, Teacher T, float t, const HeadScalars* __restrict__ S) {
    const uint32_t top = SOFT ? T.top : 0, per = top + 1, count = S->count;
    for (uint64_t at = (uint64_t)blockIdx.x * 256 + threadIdx.x; at < (uint64_t)count * per; at += (uint64_t)gridDim.x * 256) {
        const uint32_t row = at / per, k = at % per;
        const int32_t label = R.label[row];
        const size_t from = SOFT ? (size_t)R.token[row] * top : 0;
        const int32_t j = SOFT && k < top ? T.index[from + k] : label;
        if (j < 0 || (uint32_t)j - G.first >= G.n) continue;
        const RowGradient g = row_gradient(R, row, S->most, t, SOFT);
        const float z = SOFT && k < top ? T.z[(size_t)row * top + k] : R.z_label[row];
        float q = 0.0f;
        bool listed = false;
        for (uint32_t v = 0; v < top; ++v)
            if (T.index[from + v] == j) q += T.q[from + v], listed = true;
        if (k == top && listed) continue;                  // an entry of the teacher's is the label: it writes for both
        float d = SOFT ? g.softmaxes(z) - g.c2 * q : g.c1 * exp_of(z - g.lse);
        if (j == label) d -= g.c1;
        uint16_t hi, lo;
        put_dz<E, F32>(d, &hi, &lo);
        const size_t to = (size_t)row * G.ld + ((uint32_t)j - G.first);
        G.hi[to] = hi;
        if (F32) G.lo[to] = lo;
    }
}

// ------------------------------------------------------------------ gradients

// dH, partial sums: workgroups of split s take a stretch of the piece's vocabulary.  sums: [splits, rows, ld].
template <class E, int BP, int BQ, int WP, int WQ>
__global__ void __launch_bounds__(WP * WQ * 64) k_head_dh(Operand W, Operand G, uint32_t splits, uint32_t per_split,
                                                          float* __restrict__ sums, uint32_t ld, bool add,
                                                          const HeadScalars* __restrict__ S) {
    typedef Product<E, BP, BQ, WP, WQ, true, false> M;
    __shared__ __align__(1024) char lds[M::LDS];
    const uint32_t count = S->count, rows = G.extent, np = (W.extent + BP - 1) / BP, nq = rows / BQ;
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

enum OutType { OUT_F32, OUT_BF16, OUT_F16 };
template <int OUT>
__device__ __forceinline__ void put(void* out, int64_t at, float x) {
    if (OUT == OUT_F32) static_cast<float*>(out)[at] = x;
    else static_cast<uint16_t*>(out)[at] = OUT == OUT_BF16 ? Bf16::bits(x) : F16::bits(x);
}

// dH: the splits' sums in order, times what dz and W were scaled by, to the token's row; zeros for tokens that do not count.
template <int OUT, bool F32>
__global__ void __launch_bounds__(256) k_head_dh_out(const float* __restrict__ sums, uint32_t splits, uint32_t rows, uint32_t ld,
                                                     HeadRows R, uint32_t dim, float scale, void* __restrict__ dh, int64_t ld_dh,
                                                     const HeadScalars* __restrict__ S) {
    const uint32_t token = blockIdx.x;
    const int32_t row = R.row[token];
    const float factor = scale * S->most * (1.0f / DZ_SCALE), s = F32 ? 1.0f / split_scale(S->w_max) : 1.0f;
    for (uint32_t c = threadIdx.x; c < dim; c += 256) {
        float x = 0.0f;
        if (row >= 0) {
            for (uint32_t v = 0; v < splits; ++v) x += sums[((size_t)v * rows + row) * ld + c];
            x = x * s * factor;
        }
        put<OUT>(dh, token * ld_dh + c, x);
    }
}

// dW of a piece: rows of the vocabulary, summed over the rows of tokens.  wide_rows: every row of dw is 4-byte aligned.
template <class E, int BP, int BQ, int WP, int WQ, int OUT, bool F32>
__global__ void __launch_bounds__(WP * WQ * 64) k_head_dw(Operand H, Operand G, float scale, void* __restrict__ dw, int64_t ld_dw,
                                                          bool wide_rows, uint32_t first, uint32_t dim, const HeadScalars* __restrict__ S) {
    typedef Product<E, BP, BQ, WP, WQ, true, true> M;
    __shared__ __align__(1024) char lds[M::LDS];
    const uint32_t count = S->count, n = G.extent;
    uint32_t tp, tq;
    tile_of(blockIdx.x, (dim + BP - 1) / BP, (n + BQ - 1) / BQ, &tp, &tq);
    const uint32_t k_end = (count + BK - 1) & ~(BK - 1);
    H.summed = G.summed = k_end;
    M mm;
    mm.run(H, G, tp * BP, tq * BQ, 0, k_end, lds);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t p0 = tp * BP + M::p_of(wave), q0 = tq * BQ + M::q_of(wave);
    const float factor = scale * S->most * (1.0f / DZ_SCALE), s = F32 ? 1.0f / split_scale(S->h_max) : 1.0f;
    typedef Rows32<OUT == OUT_F32 ? 4 : 2> Out;
    static_assert(BP / WP == Out::ENTRIES && M::WAVES * Out::BYTES <= M::LDS, "a wavefront's rows");
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
        // 128-bit stores need no more than 4-byte alignment
        Out::each(mine, lane, [&](uint32_t row, uint32_t p, uint4 v) {
            const uint32_t q = q0 + b * 32 + row;
            if (q >= n || p0 + p >= dim) return;
            char* to = static_cast<char*>(dw) + ((int64_t)(first + q) * ld_dw + p0 + p) * SIZE;
            if (p0 + p + Out::PER_CHUNK <= dim && (OUT == OUT_F32 || wide_rows)) {
                typedef uint32_t quad_any __attribute__((ext_vector_type(4), aligned(4)));
                *reinterpret_cast<quad_any*>(to) = quad_any{v.x, v.y, v.z, v.w};
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
