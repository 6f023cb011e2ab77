// Kernels of the expert balance: softmax of a router's logits summed over tokens, counts of the experts' slots, and the gradient of
// the loss that ties them together.  With N tokens that count, p = softmax(x), L = log sum exp x, share_e = counts_e / (N slots):
//   loss0 = E sum_e share_e (1 / N) sum_i p_ie,  loss1 = (1 / N) sum_i L_i^2
//   dx_ij = p_ij (balance E / N (share_j - sum_e p_ie share_e) + 2 z / N L_i)
// The counts are needed before the first gradient, so the logits are read twice; the second time they come from the memory-side
// cache where they fit.  131072 tokens x 256 experts in binary32 (134 MB): sums 41 us (3.3 TB/s), joining the workgroups' sums 6,
// gradient 50 (5.4 TB/s read and written).  With a wavefront per token, which takes six steps to a sum instead of four and a
// quarter of the tokens to a step, the sums took 102 us.  16384 x 64 in bf16: 5 + 5 + 5 us, launches for the most part.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/iwp_losses.h"
#include "iwp_head.hpp"

namespace iwp {

struct BalanceSums {
    float* p;              // [workgroups, experts] sums of p
    uint32_t* slots;       // [workgroups, experts]
    float* square;         // [workgroups] sums of L^2
    uint32_t* tokens;      // [workgroups] tokens that count
    float* p_all;          // [experts]
    float* square_all;
    uint32_t* tokens_all;
};

// exp(d) 2^40 for d <= 0, a normal number down to exp(d) of 2^-166: the gradient, which is proportional to it, is rounded once.
__device__ __forceinline__ float exp_raised(float d) {
    const float t = fmaxf(d * LOG2E, -300.0f), n = rintf(t);
    return ldexpf(exp2_fast(t - n), (int)n + 40);
}

// A token's experts over `lanes` lanes (a power of two), CHUNKS times 16 bytes each: chunk c of lane l starts at expert
// (c lanes + l) WIDTH.  A wavefront has 64 / lanes tokens at a time.
template <int IN, int CHUNKS>
struct TokenLanes {
    static constexpr int WIDTH = IN == OUT_F32 ? 4 : 8, N = CHUNKS * WIDTH;
    uint32_t experts, lanes, lane, of;                 // of: which of the wavefront's tokens
    __device__ __forceinline__ TokenLanes(uint32_t experts, uint32_t lanes) : experts(experts), lanes(lanes) {
        lane = threadIdx.x & (lanes - 1);
        of = (threadIdx.x & 63) / lanes;
    }
    __device__ __forceinline__ uint32_t tokens() const { return 64 / lanes; }
    __device__ __forceinline__ uint32_t first(int c) const { return (c * lanes + lane) * WIDTH; }
    __device__ __forceinline__ uint32_t expert(int i) const { return first(i / WIDTH) + i % WIDTH; }

    __device__ __forceinline__ void load(const void* x, int64_t at, words4 (&v)[CHUNKS]) const {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const uint32_t e0 = first(c);
            if (IN == OUT_F32) {
                const float* p = static_cast<const float*>(x) + at + e0;
                if (e0 + WIDTH <= experts) {
                    v[c] = *reinterpret_cast<const words4*>(p);
                } else {
#pragma unroll
                    for (uint32_t e = 0; e < 4; ++e) v[c][e] = e0 + e < experts ? __float_as_uint(p[e]) : 0xff800000u;
                }
            } else {
                const uint16_t* p = static_cast<const uint16_t*>(x) + at + e0;
                const uint32_t none = IN == OUT_BF16 ? 0xff80u : 0xfc00u;              // -inf
                if (e0 + WIDTH <= experts) {
                    v[c] = (words4)*reinterpret_cast<const words4_any*>(p);
                } else {
#pragma unroll
                    for (uint32_t e = 0; e < 8; e += 2)
                        v[c][e / 2] = (e0 + e < experts ? p[e] : none) | (e0 + e + 1 < experts ? p[e + 1] : none) << 16;
                }
            }
        }
    }
    static __device__ __forceinline__ void unpack(const words4 (&v)[CHUNKS], float (&y)[N]) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (IN == OUT_F32) y[i] = __uint_as_float(v[i / 4 % CHUNKS][i % 4]);
            else {
                const uint16_t b = (uint16_t)(v[i / 8 % CHUNKS][i % 8 / 2] >> (i % 2 * 16));
                y[i] = IN == OUT_BF16 ? Bf16::value(b) : F16::value(b);
            }
        }
    }
    __device__ __forceinline__ void store(void* out, int64_t at, const float (&y)[N]) const {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const uint32_t e0 = first(c);
            words4 v;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                if (IN == OUT_F32) v[w] = __float_as_uint(y[c * WIDTH % N + w]);
                else {
                    const float a = y[(c * WIDTH + 2 * w) % N], b = y[(c * WIDTH + 2 * w + 1) % N];
                    v[w] = IN == OUT_BF16 ? Bf16::bits(a) | (uint32_t)Bf16::bits(b) << 16 : F16::bits(a) | (uint32_t)F16::bits(b) << 16;
                }
            }
            if (e0 + WIDTH <= experts) {
                if (IN == OUT_F32) *reinterpret_cast<words4*>(static_cast<float*>(out) + at + e0) = v;
                else *reinterpret_cast<words4_any*>(static_cast<uint16_t*>(out) + at + e0) = v;
            } else {
#pragma unroll
                for (int e = 0; e < WIDTH; ++e)
                    if (e0 + e < experts) put<IN>(out, at + e0 + e, y[c * WIDTH + e]);
            }
        }
    }
    __device__ __forceinline__ float sum(float s) const {
        for (uint32_t o = lanes / 2; o; o >>= 1) s += __shfl_xor(s, o);
        return s;
    }
    // A token's exponentials in place of its logits, what they take to be probabilities, its L; false where all logits are -inf.
    __device__ __forceinline__ bool softmax(float (&x)[N], float* by, float* log_sum) const {
        float m = -INFINITY;
#pragma unroll
        for (int i = 0; i < N; ++i) m = x[i] != x[i] ? INFINITY : fmaxf(m, x[i]);    // NaN as infinity: the whole token is NaN
        for (uint32_t o = lanes / 2; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
        float s = 0.0f;
        const float from = m == -INFINITY ? 0.0f : m;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            x[i] = exp_raised(x[i] - from);
            s += x[i];
        }
        s = sum(s);
        *by = 1.0f / s;
        *log_sum = m + logf(s * 0x1p-40f);
        return m != -INFINITY;
    }
};

struct Router {
    const void* x;
    int64_t ld;
    uint32_t tokens, experts, lanes, slots;
    const int32_t* chosen;
    const uint8_t* keep;
};
struct BalanceGradient {
    float balance, z;
    void* dx;
    int64_t ld;
};

// Sums over the tokens that wavefront `wave` of `waves` takes.
template <int IN, int CHUNKS>
__device__ __forceinline__ void balance_sums(const Router& r, uint32_t wave, uint32_t waves, uint32_t* of_expert,
                                             float (&p)[TokenLanes<IN, CHUNKS>::N], float* square, uint32_t* n) {
    typedef TokenLanes<IN, CHUNKS> L;
    const L l(r.experts, r.lanes);
    const uint32_t at_once = l.tokens(), stride = waves * at_once;
    words4 next[CHUNKS] = {};
    bool next_in = false;
    uint32_t i = wave * at_once + l.of;
    auto request = [&](uint32_t i) {
        next_in = i < r.tokens && !(r.keep && !r.keep[i]);
        if (next_in) l.load(r.x, (int64_t)i * r.ld, next);
    };
    request(i);
    for (uint32_t base = wave * at_once; base < r.tokens; base += stride, i += stride) {
        words4 now[CHUNKS];
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) now[c] = next[c];
        bool in = next_in;
        request(i + stride);
        float y[L::N], by, log_sum;
        L::unpack(now, y);
        in = l.softmax(y, &by, &log_sum) && in;
        if (!in) continue;
#pragma unroll
        for (int v = 0; v < L::N; ++v) p[v] += y[v] * by;
        if (l.lane == 0) {
            *square += log_sum * log_sum;
            ++*n;
        }
        for (uint32_t k = l.lane; k < r.slots; k += r.lanes) {
            const uint32_t e = r.chosen[(size_t)i * r.slots + k];
            if (e < r.experts) atomicAdd(&of_expert[e], 1u);
        }
    }
    // over the wavefront's tokens
    for (uint32_t o = r.lanes; o < 64; o <<= 1) {
#pragma unroll
        for (int v = 0; v < L::N; ++v) p[v] += __shfl_xor(p[v], o);
        *square += __shfl_xor(*square, o);
        *n += __shfl_xor(*n, o);
    }
}

// The gradient of the tokens that wavefront `wave` of `waves` takes.
template <int IN, int CHUNKS, class Share>
__device__ __forceinline__ void balance_gradient(const Router& r, const BalanceGradient& g, uint32_t wave, uint32_t waves, float by_n, Share share_of) {
    typedef TokenLanes<IN, CHUNKS> L;
    const L l(r.experts, r.lanes);
    const uint32_t at_once = l.tokens(), stride = waves * at_once;
    float share[L::N];
#pragma unroll
    for (int v = 0; v < L::N; ++v) share[v] = l.expert(v) < r.experts ? share_of(l.expert(v)) : 0.0f;
    const float cb = g.balance * (float)r.experts * by_n, cz = 2.0f * g.z * by_n;
    words4 next[CHUNKS] = {};
    bool next_in = false;
    uint32_t i = wave * at_once + l.of;
    auto request = [&](uint32_t i) {
        next_in = i < r.tokens && !(r.keep && !r.keep[i]);
        if (next_in) l.load(r.x, (int64_t)i * r.ld, next);
    };
    request(i);
    for (uint32_t base = wave * at_once; base < r.tokens; base += stride, i += stride) {
        words4 now[CHUNKS];
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) now[c] = next[c];
        bool in = next_in;
        request(i + stride);
        float y[L::N], by, log_sum, inner = 0.0f;
        L::unpack(now, y);
        in = l.softmax(y, &by, &log_sum) && in;
#pragma unroll
        for (int v = 0; v < L::N; ++v) inner += y[v] * share[v];
        inner = l.sum(inner) * by;
#pragma unroll
        for (int v = 0; v < L::N; ++v) y[v] = in ? y[v] * (by * (cb * (share[v] - inner) + cz * log_sum)) : 0.0f;
        if (i < r.tokens) l.store(g.dx, (int64_t)i * g.ld, y);
    }
}

template <int IN, int CHUNKS>
__global__ void __launch_bounds__(256) k_balance_rows(Router r, BalanceSums B) {
    typedef TokenLanes<IN, CHUNKS> L;
    __shared__ uint32_t of_expert[IWP_MAX_EXPERTS];
    __shared__ float sums[4][IWP_MAX_EXPERTS];
    __shared__ float squares[4];
    __shared__ uint32_t counted[4];
    const uint32_t wave = threadIdx.x >> 6;
    for (uint32_t e = threadIdx.x; e < r.experts; e += 256) of_expert[e] = 0;
    __syncthreads();
    float p[L::N] = {}, square = 0.0f;
    uint32_t n = 0;
    balance_sums<IN, CHUNKS>(r, blockIdx.x * 4 + wave, gridDim.x * 4, of_expert, p, &square, &n);
    const L l(r.experts, r.lanes);
    if (l.of == 0) {
#pragma unroll
        for (int v = 0; v < L::N; ++v)
            if (l.expert(v) < r.experts) sums[wave][l.expert(v)] = p[v];
    }
    if ((threadIdx.x & 63) == 0) squares[wave] = square, counted[wave] = n;
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < r.experts; e += 256) {
        B.p[(size_t)blockIdx.x * r.experts + e] = (sums[0][e] + sums[1][e]) + (sums[2][e] + sums[3][e]);
        B.slots[(size_t)blockIdx.x * r.experts + e] = of_expert[e];
    }
    if (threadIdx.x == 0) {
        B.square[blockIdx.x] = (squares[0] + squares[1]) + (squares[2] + squares[3]);
        B.tokens[blockIdx.x] = counted[0] + counted[1] + counted[2] + counted[3];
    }
}

// A wavefront per expert, and one for the squares; workgroups' sums in a fixed order.
__global__ void __launch_bounds__(256) k_balance_join(BalanceSums B, uint32_t groups, uint32_t experts, int32_t* __restrict__ counts) {
    const uint32_t e = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (e > experts) return;
    float s = 0.0f;
    uint32_t n = 0;
#pragma unroll 4
    for (uint32_t g = lane; g < groups; g += 64) {
        s += e < experts ? B.p[(size_t)g * experts + e] : B.square[g];
        n += e < experts ? B.slots[(size_t)g * experts + e] : B.tokens[g];
    }
    for (int o = 32; o; o >>= 1) {
        s += __shfl_xor(s, o);
        n += __shfl_xor(n, o);
    }
    if (lane) return;
    if (e < experts) B.p_all[e] = s, counts[e] = (int32_t)n;
    else *B.square_all = s, *B.tokens_all = n;
}

// The first wavefront of a launch: loss[0] from the experts' slots and sums, loss[1].
template <class Slots, class Sum>
__device__ __forceinline__ void balance_loss(uint32_t experts, uint32_t slots, uint32_t n, float square, Slots slots_of, Sum p_of, float* loss) {
    const uint32_t lane = threadIdx.x & 63;
    const float by_n = n ? 1.0f / (float)n : 0.0f;
    float s = 0.0f;
    for (uint32_t e = lane; e < experts; e += 64) s += (float)slots_of(e) / (float)slots * by_n * (p_of(e) * by_n);
    for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
    if (lane == 0) {
        loss[0] = (float)experts * s;
        loss[1] = square * by_n;
    }
}

// The gradient; the first wavefront also has the losses.
template <int IN, int CHUNKS>
__global__ void __launch_bounds__(256) k_balance_grad(Router r, BalanceGradient g, BalanceSums B, const int32_t* __restrict__ counts,
                                                      float* __restrict__ loss) {
    const uint32_t n = *B.tokens_all;
    const float by_n = n ? 1.0f / (float)n : 0.0f;
    if (blockIdx.x == 0 && threadIdx.x < 64)
        balance_loss(r.experts, r.slots, n, *B.square_all, [&](uint32_t e) { return counts[e]; }, [&](uint32_t e) { return B.p_all[e]; }, loss);
    if (g.dx)
        balance_gradient<IN, CHUNKS>(r, g, blockIdx.x * 4 + (threadIdx.x >> 6), gridDim.x * 4, by_n,
                                     [&](uint32_t e) { return (float)counts[e] / (float)r.slots * by_n; });
}

// All of it in one workgroup, for small batches.
constexpr uint32_t BALANCE_ONE_WAVES = 16;
template <int IN, int CHUNKS>
__global__ void __launch_bounds__(BALANCE_ONE_WAVES * 64) k_balance_one(Router r, BalanceGradient g, int32_t* __restrict__ counts,
                                                                        float* __restrict__ loss) {
    typedef TokenLanes<IN, CHUNKS> L;
    constexpr uint32_t THREADS = BALANCE_ONE_WAVES * 64;
    __shared__ uint32_t of_expert[IWP_MAX_EXPERTS];
    __shared__ float sums[BALANCE_ONE_WAVES][IWP_MAX_EXPERTS];
    __shared__ float squares[BALANCE_ONE_WAVES];
    __shared__ uint32_t counted[BALANCE_ONE_WAVES];
    const uint32_t wave = threadIdx.x >> 6;
    for (uint32_t e = threadIdx.x; e < r.experts; e += THREADS) of_expert[e] = 0;
    __syncthreads();
    float p[L::N] = {}, square = 0.0f;
    uint32_t n = 0;
    balance_sums<IN, CHUNKS>(r, wave, BALANCE_ONE_WAVES, of_expert, p, &square, &n);
    const L l(r.experts, r.lanes);
    if (l.of == 0) {
#pragma unroll
        for (int v = 0; v < L::N; ++v)
            if (l.expert(v) < r.experts) sums[wave][l.expert(v)] = p[v];
    }
    if ((threadIdx.x & 63) == 0) squares[wave] = square, counted[wave] = n;
    __syncthreads();
    n = 0;
    square = 0.0f;
    for (uint32_t v = 0; v < BALANCE_ONE_WAVES; ++v) n += counted[v], square += squares[v];
    for (uint32_t e = threadIdx.x; e < r.experts; e += THREADS) counts[e] = (int32_t)of_expert[e];
    if (threadIdx.x < 64) {
        balance_loss(r.experts, r.slots, n, square, [&](uint32_t e) { return of_expert[e]; },
                     [&](uint32_t e) {
                         float s = 0.0f;
                         for (uint32_t v = 0; v < BALANCE_ONE_WAVES; ++v) s += sums[v][e];
                         return s;
                     }, loss);
    }
    const float by_n = n ? 1.0f / (float)n : 0.0f;
    if (g.dx)
        balance_gradient<IN, CHUNKS>(r, g, wave, BALANCE_ONE_WAVES, by_n, [&](uint32_t e) { return (float)of_expert[e] / (float)r.slots * by_n; });
}

}  // namespace iwp
