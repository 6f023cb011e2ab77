// Kernels of the choice of experts and of its gradient.  A token's experts lie over a part of a wavefront as in the expert balance
// (TokenLanes), so the logits are read once, and everything about a token happens between its lanes:
//   c = score + bias in binary64, or the logits themselves where their order is the scores' order (no bias, no sums over groups);
//   groups: best one or two c of every group by way of LDS, a group's rank by counting;
//   then slot after slot the largest c that is left, found by every lane among its own and between lanes in log2(lanes) steps.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/iwp_experts.h"
#include "iwp_tokens.hpp"

namespace iwp {

struct RouteCall {
    const void* x;
    int64_t ld;
    uint32_t tokens, experts, lanes, slots;
    const float* bias;
    bool sigmoid, renormalise;
    uint32_t groups, top_groups, group_top;
    float scale;
    const uint8_t* keep;
    int32_t* chosen;
    float* weight;
};

// e^(min(x, 0) - m) / (1 + e^-|x|) for m >= min(x, 0): a sigmoid over e^m, which does not vanish where all a token's sigmoids are small.
__device__ __forceinline__ float sigmoid_over(float x, float m) { return expf(fminf(x, 0.0f) - m) / (1.0f + expf(-fabsf(x))); }

// A part of a wavefront that has one token.
struct Part {
    uint32_t lanes;
    template <class F, class T>
    __device__ __forceinline__ T reduce(T v, F f) const {
        for (uint32_t o = lanes / 2; o; o >>= 1) v = f(v, __shfl_xor(v, o));
        return v;
    }
    __device__ __forceinline__ float sum(float v) const { return reduce(v, [](float a, float b) { return a + b; }); }
    __device__ __forceinline__ double sum(double v) const { return reduce(v, [](double a, double b) { return a + b; }); }
    __device__ __forceinline__ float max(float v) const { return reduce(v, [](float a, float b) { return fmaxf(a, b); }); }
    __device__ __forceinline__ bool any(bool v) const { return reduce((int)v, [](int a, int b) { return a | b; }) != 0; }
};

struct Slot {              // what a slot got, in LDS until the token's weights are known
    int32_t expert;
    float x;
};

// C: the type of c, float where the logits themselves are compared, else double.
template <int IN, int CHUNKS, class C, bool GROUPS>
__global__ void __launch_bounds__(256) k_route(RouteCall r) {
    typedef TokenLanes<IN, CHUNKS> L;
    constexpr bool BY_SCORE = sizeof(C) == 8;
    constexpr C NONE = -(C)INFINITY;
    extern __shared__ __align__(16) char shared[];
    const L l(r.experts, r.lanes);
    const Part part{r.lanes};
    const uint32_t wave = threadIdx.x >> 6, at_once = l.tokens(), tokens = (blockDim.x >> 6) * at_once;      // of the workgroup at a time
    const uint32_t mine = wave * at_once + l.of;
    Slot* slot = reinterpret_cast<Slot*>(shared) + (size_t)mine * r.slots;
    C* row = reinterpret_cast<C*>(shared + (size_t)tokens * r.slots * sizeof(Slot)) + (size_t)mine * (r.experts + r.groups);
    C* of_group = row + r.experts;
    for (uint32_t base = blockIdx.x * tokens; base < r.tokens; base += gridDim.x * tokens) {
        const uint32_t i = base + mine;
        const bool in = i < r.tokens && !(r.keep && !r.keep[i]);
        words4 raw[CHUNKS] = {};
        if (in) l.load(r.x, (int64_t)i * r.ld, raw);
        float x[L::N];
        L::unpack(raw, x);
        bool nan = false;
        float m = -INFINITY;
        C c[L::N];
#pragma unroll
        for (int v = 0; v < L::N; ++v) {
            if (!in || l.expert(v) >= r.experts) x[v] = -INFINITY;
            nan |= x[v] != x[v];
            if (x[v] != x[v]) x[v] = -INFINITY;
            m = fmaxf(m, x[v]);
        }
        m = part.max(m);
        nan = part.any(nan) || (!r.sigmoid && m == INFINITY);
        const float from = m == -INFINITY ? 0.0f : m;
        float by = 1.0f;                                                            // softmax: 1 / sum of e^(x - m)
        if (BY_SCORE) {
            double e[L::N], sum = 0.0;
#pragma unroll
            for (int v = 0; v < L::N; ++v) {
                e[v] = r.sigmoid ? 1.0 / (1.0 + exp(-(double)x[v])) : exp((double)x[v] - (double)from);
                sum += e[v];
            }
            sum = part.sum(sum);
            by = (float)(1.0 / sum);
#pragma unroll
            for (int v = 0; v < L::N; ++v) {
                const uint32_t ex = l.expert(v);
                double s = r.sigmoid ? e[v] : e[v] / sum;
                if (r.bias && ex < r.experts) s += (double)r.bias[ex];
                c[v] = x[v] == -INFINITY || s != s ? NONE : (C)s;
            }
        } else {
            if (!r.sigmoid && !r.renormalise) {
                float sum = 0.0f;
#pragma unroll
                for (int v = 0; v < L::N; ++v) sum += expf(x[v] - from);
                by = 1.0f / part.sum(sum);
            }
#pragma unroll
            for (int v = 0; v < L::N; ++v) c[v] = (C)x[v];
        }
        if (GROUPS) {
            const uint32_t size = r.experts / r.groups;
#pragma unroll
            for (int v = 0; v < L::N; ++v)
                if (l.expert(v) < r.experts) row[l.expert(v)] = c[v];
            lanes_exchange();
            for (uint32_t g = l.lane; g < r.groups; g += r.lanes) {
                C first = NONE, second = NONE;
                for (uint32_t e = 0; e < size; ++e) {
                    const C y = row[g * size + e];
                    second = y > first ? first : y > second ? y : second;
                    first = y > first ? y : first;
                }
                of_group[g] = r.group_top == 2 && second != NONE ? first + second : first;
            }
            lanes_exchange();
            for (uint32_t g = l.lane; g < r.groups; g += r.lanes) {
                const C y = of_group[g];
                uint32_t better = 0;
                for (uint32_t o = 0; o < r.groups; ++o) better += of_group[o] > y || (of_group[o] == y && o < g);
                if (better >= r.top_groups || y == NONE)
                    for (uint32_t e = 0; e < size; ++e) row[g * size + e] = NONE;
            }
            lanes_exchange();
#pragma unroll
            for (int v = 0; v < L::N; ++v) c[v] = l.expert(v) < r.experts ? row[l.expert(v)] : NONE;
            lanes_exchange();
        }
        // the slots: of equal c the lower expert, which is also the lower v of a lane
        float most = -INFINITY;                                                     // of the chosen logits (sigmoid: at most 0)
        for (uint32_t k = 0; k < r.slots; ++k) {
            C best = NONE;
            uint32_t at = 0xffffffffu;
            float logit = 0.0f;
#pragma unroll
            for (int v = 0; v < L::N; ++v)
                if (c[v] > best) best = c[v], at = l.expert(v), logit = x[v];
            for (uint32_t o = r.lanes / 2; o; o >>= 1) {
                const C other = __shfl_xor(best, o);
                const uint32_t other_at = __shfl_xor(at, o);
                const float other_logit = __shfl_xor(logit, o);
                if (other > best || (other == best && other_at < at)) best = other, at = other_at, logit = other_logit;
            }
#pragma unroll
            for (int v = 0; v < L::N; ++v)
                if (l.expert(v) == at) c[v] = NONE;
            const bool some = best != NONE;
            if (some) most = fmaxf(most, r.sigmoid ? fminf(logit, 0.0f) : logit);
            if (l.lane == 0) slot[k] = Slot{some ? (int32_t)at : -1, logit};
        }
        lanes_exchange();
        float all = 0.0f;
        auto share = [&](const Slot& s, float m) { return s.expert < 0 ? 0.0f : r.sigmoid ? sigmoid_over(s.x, m) : expf(s.x - m); };
        if (r.renormalise) {
            for (uint32_t k = l.lane; k < r.slots; k += r.lanes) all += share(slot[k], most);
            all = part.sum(all);
        }
        if (i < r.tokens)
            for (uint32_t k = l.lane; k < r.slots; k += r.lanes) {
                const Slot s = slot[k];
                float y = r.renormalise ? share(s, most) / all : r.sigmoid ? share(s, 0.0f) : share(s, m) * by;
                y = s.expert < 0 ? 0.0f : y * r.scale;
                const size_t to = (size_t)i * r.slots + k;
                r.chosen[to] = s.expert;
                r.weight[to] = nan ? NAN : y;
            }
        lanes_exchange();
    }
}

struct RouteGradient {
    const void* x;
    int64_t ld;
    uint32_t tokens, experts, lanes, slots;
    const int32_t* chosen;
    const float* dweight;
    bool sigmoid, renormalise;
    float scale;
    const uint8_t* keep;
    const void* plus;
    int64_t ld_plus;
    void* dx;
    int64_t ld_dx;
};

struct SlotGradient {
    uint32_t expert;
    float d;
};

template <int IN>
__device__ __forceinline__ float element(const void* x, int64_t at) {
    if (IN == OUT_F32) return static_cast<const float*>(x)[at];
    const uint16_t b = static_cast<const uint16_t*>(x)[at];
    return IN == OUT_BF16 ? Bf16::value(b) : F16::value(b);
}

template <int IN, int CHUNKS>
__global__ void __launch_bounds__(256) k_route_gradient(RouteGradient r) {
    typedef TokenLanes<IN, CHUNKS> L;
    extern __shared__ __align__(16) char shared[];
    const L l(r.experts, r.lanes);
    const Part part{r.lanes};
    const uint32_t wave = threadIdx.x >> 6, at_once = l.tokens(), tokens = (blockDim.x >> 6) * at_once;
    const uint32_t mine = wave * at_once + l.of;
    SlotGradient* slot = reinterpret_cast<SlotGradient*>(shared) + (size_t)mine * r.slots;
    const bool dense = !r.sigmoid && !r.renormalise;
    for (uint32_t base = blockIdx.x * tokens; base < r.tokens; base += gridDim.x * tokens) {
        const uint32_t i = base + mine;
        bool in = i < r.tokens && !(r.keep && !r.keep[i]);
        float y[L::N], by = 0.0f, m = -INFINITY, log_sum;
#pragma unroll
        for (int v = 0; v < L::N; ++v) y[v] = 0.0f;
        if (dense) {
            words4 raw[CHUNKS] = {};
            if (in) l.load(r.x, (int64_t)i * r.ld, raw);
            L::unpack(raw, y);
#pragma unroll
            for (int v = 0; v < L::N; ++v) {
                if (l.expert(v) >= r.experts) y[v] = -INFINITY;
                m = fmaxf(m, y[v]);
            }
            m = part.max(m);
            in = l.softmax(y, &by, &log_sum) && in;
        }
        auto expert_of = [&](uint32_t k) { return in ? (uint32_t)r.chosen[(size_t)i * r.slots + k] : 0xffffffffu; };
        auto logit_of = [&](uint32_t e) { return element<IN>(r.x, (int64_t)i * r.ld + e); };
        if (r.renormalise) {
            for (uint32_t k = l.lane; k < r.slots; k += r.lanes) {
                const uint32_t e = expert_of(k);
                if (e < r.experts) m = fmaxf(m, r.sigmoid ? fminf(logit_of(e), 0.0f) : logit_of(e));
            }
            m = part.max(m);
        }
        // every slot's part: its dweight times the scale, and what the sums take
        auto value_of = [&](float x) {
            return r.sigmoid ? sigmoid_over(x, r.renormalise ? m : 0.0f) : r.renormalise ? expf(x - m) : exp_raised(x - m) * by;
        };
        float all = 0.0f, inner = 0.0f;
        for (uint32_t k = l.lane; k < r.slots; k += r.lanes) {
            const uint32_t e = expert_of(k);
            if (e >= r.experts) continue;
            const float q = value_of(logit_of(e));
            all += q;
            inner += q * r.dweight[(size_t)i * r.slots + k];
        }
        inner = part.sum(inner);
        if (r.renormalise) {
            all = part.sum(all);
            inner = inner / all;
        }
        for (uint32_t k = l.lane; k < r.slots; k += r.lanes) {
            const uint32_t e = expert_of(k);
            float d = 0.0f;
            if (e < r.experts) {
                const float x = logit_of(e), dw = r.dweight[(size_t)i * r.slots + k];
                d = dense ? dw : r.renormalise ? value_of(x) / all * (dw - inner) : value_of(x) * dw;
                if (r.sigmoid) d *= sigmoid_over(-x, 0.0f);
                d *= r.scale;
            }
            slot[k] = SlotGradient{e, d};
        }
        lanes_exchange();
        float d[L::N];
#pragma unroll
        for (int v = 0; v < L::N; ++v) d[v] = 0.0f;
        for (uint32_t k = 0; k < r.slots; ++k) {
            const SlotGradient s = slot[k];
#pragma unroll
            for (int v = 0; v < L::N; ++v) d[v] += l.expert(v) == s.expert ? s.d : 0.0f;
        }
        lanes_exchange();
        if (i >= r.tokens) continue;
        float plus[L::N];
#pragma unroll
        for (int v = 0; v < L::N; ++v) plus[v] = 0.0f;
        if (r.plus) {
            words4 raw[CHUNKS];
            l.load(r.plus, (int64_t)i * r.ld_plus, raw);
            L::unpack(raw, plus);
        }
#pragma unroll
        for (int v = 0; v < L::N; ++v) {
            const float g = dense ? y[v] * by * (d[v] - inner * r.scale) : d[v];
            y[v] = in ? plus[v] + g : plus[v];
        }
        l.store(r.dx, (int64_t)i * r.ld_dx, y);
    }
}

}  // namespace iwp
