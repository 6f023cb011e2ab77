// Kernels of the expert balance: softmax of a router's logits summed over tokens, counts of the experts' slots, and the gradient of
// the loss that ties them together.  With N tokens that count, p = softmax(x), L = log sum exp x, share_e = counts_e / (N slots):
//   loss0 = E sum_e share_e (1 / N) sum_i p_ie,  loss1 = (1 / N) sum_i L_i^2
//   dx_ij = p_ij (balance E / N (share_j - sum_e p_ie share_e) + 2 z / N L_i)
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

template <int IN>
__device__ __forceinline__ float router_logit(const void* x, int64_t at) {
    if (IN == OUT_F32) return static_cast<const float*>(x)[at];
    const uint16_t b = static_cast<const uint16_t*>(x)[at];
    return IN == OUT_BF16 ? Bf16::value(b) : F16::value(b);
}

// exp(d) 2^40 for d <= 0, a normal number down to exp(d) of 2^-166: the gradient, which is proportional to it, is rounded once.
__device__ __forceinline__ float exp_raised(float d) {
    const float t = fmaxf(d * LOG2E, -300.0f), n = rintf(t);
    return ldexpf(exp2_fast(t - n), (int)n + 40);
}

// One token: its exponentials in place of its logits (lane + 64 v), what they take to be probabilities, its L; false if it does not
// count.
template <int NV>
__device__ __forceinline__ bool token_softmax(float (&x)[NV], float* by, float* log_sum) {
    float m = -INFINITY;
    bool nan = false;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        nan |= x[v] != x[v];
        m = fmaxf(m, x[v]);
    }
    for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    if (__ballot(nan)) m = NAN;
    if (m == -INFINITY) return false;
    float s = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        x[v] = exp_raised(x[v] - m);
        s += x[v];
    }
    for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
    *by = 1.0f / s;
    *log_sum = m + logf(s * 0x1p-40f);
    return true;
}

template <int IN, int NV>
__device__ __forceinline__ void token_logits(const void* x, int64_t row, uint32_t experts, int lane, float (&out)[NV]) {
#pragma unroll
    for (int v = 0; v < NV; ++v) out[v] = lane + 64 * v < (int)experts ? router_logit<IN>(x, row + lane + 64 * v) : -INFINITY;
}

template <int IN, int NV>
__global__ void __launch_bounds__(256) k_balance_rows(const void* __restrict__ x, int64_t ld, uint32_t tokens, uint32_t experts,
                                                      const int32_t* __restrict__ chosen, uint32_t slots,
                                                      const uint8_t* __restrict__ keep, BalanceSums B) {
    __shared__ uint32_t of_expert[IWP_MAX_EXPERTS];
    __shared__ float sums[4][64 * NV];
    __shared__ float squares[4];
    __shared__ uint32_t counted[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (uint32_t e = threadIdx.x; e < experts; e += 256) of_expert[e] = 0;
    __syncthreads();
    float p[NV] = {}, square = 0.0f;
    uint32_t n = 0;
    for (uint32_t i = blockIdx.x * 4 + wave; i < tokens; i += gridDim.x * 4) {
        if (keep && !keep[i]) continue;
        float y[NV], by, log_sum;
        token_logits<IN, NV>(x, (int64_t)i * ld, experts, lane, y);
        if (!token_softmax<NV>(y, &by, &log_sum)) continue;
#pragma unroll
        for (int v = 0; v < NV; ++v) p[v] += y[v] * by;
        square += log_sum * log_sum;
        ++n;
        for (uint32_t k = lane; k < slots; k += 64) {
            const uint32_t e = chosen[(size_t)i * slots + k];
            if (e < experts) atomicAdd(&of_expert[e], 1u);
        }
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) sums[wave][lane + 64 * v] = p[v];
    if (lane == 0) squares[wave] = square, counted[wave] = n;
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < experts; e += 256) {
        B.p[(size_t)blockIdx.x * experts + e] = (sums[0][e] + sums[1][e]) + (sums[2][e] + sums[3][e]);
        B.slots[(size_t)blockIdx.x * experts + e] = of_expert[e];
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

// The gradient, a wavefront per token; the first workgroup also has the losses.
template <int IN, int NV>
__global__ void __launch_bounds__(256) k_balance_grad(const void* __restrict__ x, int64_t ld, uint32_t tokens, uint32_t experts,
                                                      uint32_t slots, const uint8_t* __restrict__ keep, float balance, float z,
                                                      BalanceSums B, const int32_t* __restrict__ counts, float* __restrict__ loss,
                                                      void* __restrict__ dx, int64_t ld_dx) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t n = *B.tokens_all;
    const float by_n = n ? 1.0f / (float)n : 0.0f;
    float share[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v)
        share[v] = lane + 64 * v < (int)experts && n ? (float)counts[lane + 64 * v] / ((float)n * (float)slots) : 0.0f;
    if (blockIdx.x == 0 && wave == 0) {
        float s = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
            if (lane + 64 * v < (int)experts) s += share[v] * (B.p_all[lane + 64 * v] * by_n);
        for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
        if (lane == 0) {
            loss[0] = (float)experts * s;
            loss[1] = *B.square_all * by_n;
        }
    }
    if (!dx) return;
    const float cb = balance * (float)experts * by_n, cz = 2.0f * z * by_n;
    for (uint32_t i = blockIdx.x * 4 + wave; i < tokens; i += gridDim.x * 4) {
        float y[NV], by = 0.0f, log_sum = 0.0f, inner = 0.0f;
        bool in = !(keep && !keep[i]);
        if (in) {
            token_logits<IN, NV>(x, (int64_t)i * ld, experts, lane, y);
            in = token_softmax<NV>(y, &by, &log_sum);
        }
        if (in) {
#pragma unroll
            for (int v = 0; v < NV; ++v) inner += y[v] * share[v];
            for (int o = 32; o; o >>= 1) inner += __shfl_xor(inner, o);
            inner *= by;
        }
#pragma unroll
        for (int v = 0; v < NV; ++v)
            if (lane + 64 * v < (int)experts)
                put<IN>(dx, (int64_t)i * ld_dx + lane + 64 * v, in ? y[v] * (by * (cb * (share[v] - inner) + cz * log_sum)) : 0.0f);
    }
}

}  // namespace iwp
