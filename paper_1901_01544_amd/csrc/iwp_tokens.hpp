// How a router's logits lie over lanes: a token's experts in a part of a wavefront, several tokens to a wavefront.  What the expert
// balance and the routing share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "iwp_matrix.hpp"

namespace iwp {

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

}  // namespace iwp
