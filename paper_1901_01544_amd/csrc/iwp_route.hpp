// Kernels of the choice of experts and of its gradient.  A token's experts lie over a part of a wavefront as in the expert balance
// (TokenLanes), so the logits are read once, and everything about a token happens between its lanes:
//   c = score + bias, or without a bias the logits themselves, in whose order the scores are (sums over groups are of scores all the same);
//   groups: best one or two c of every group between the lanes that have it, a group's rank by counting;
//   slots: the largest c that is left, one after the other, or where there are many lanes all at once (see candidates).
// Scores decide in binary64, but are computed in binary32 first: where no two c that the choice depends on are closer than twice what
// binary32 may be off, it is the choice.  Else the wavefront does the token again in binary64, value by value in LDS.  That is 6 of 10000 tokens of the
// case below (81 by softmax), 71 (154) in bf16 with its biases of 81 values.  Scores that are equal are close as well: with one bias for all experts a third of
// the tokens in bf16, 5 % in fp16, and every token of a router whose logits are all alike.
//
// Bound by instructions where experts are many.  131072 tokens x 256 experts in binary32, 8 slots: by logits alone 28 to 30 us, which is reading them
// (134 MB, 4.5 TB/s); sigmoid scores with a bias 51; of 4 of 8 groups by their best two 76 to 79, 1258 vector instructions a wavefront of four tokens, which
// the vector units issue in all cycles; without a bias 65.  In bf16 98, without a bias 70, with a bias of zeros 270 to 281; logits all alike 455.  In binary64
// throughout 264; slots one after the other instead of all at once 120.
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

template <int IN>
__device__ __forceinline__ float element(const void* x, int64_t at) {
    if (IN == OUT_F32) return static_cast<const float*>(x)[at];
    const uint16_t b = static_cast<const uint16_t*>(x)[at];
    return IN == OUT_BF16 ? Bf16::value(b) : F16::value(b);
}

// A part of a wavefront that has one token: `lanes`, a power of two.  LANES: that number where it is known to the compiler, else 0.
template <int LANES>
struct PartOf {
    uint32_t lanes;
    __device__ __forceinline__ PartOf(uint32_t lanes) : lanes(LANES ? LANES : lanes) {}
    template <int CONTROL, class T>
    static __device__ __forceinline__ T moved(T v) {
        return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CONTROL, 0xf, 0xf, true));
    }
    // f over all lanes, in every lane: neighbours, pairs, quads (mirrored, whose lanes hold the same by then), rows of 16
    template <class F, class T>
    __device__ __forceinline__ T reduce(T v, F f) const {
        if (lanes > 1) v = f(v, moved<0xb1>(v));                                    // quad_perm 1 0 3 2
        if (lanes > 2) v = f(v, moved<0x4e>(v));                                    // quad_perm 2 3 0 1
        if (lanes > 4) v = f(v, moved<0x141>(v));                                   // row_half_mirror
        if (lanes > 8) v = f(v, moved<0x140>(v));                                   // row_mirror
        if (lanes > 16) v = f(v, (T)__shfl_xor(v, 16));
        if (lanes > 32) v = f(v, (T)__shfl_xor(v, 32));
        return v;
    }
    __device__ __forceinline__ float sum(float v) const { return reduce(v, [](float a, float b) { return a + b; }); }
    __device__ __forceinline__ float max(float v) const { return reduce(v, [](float a, float b) { return fmaxf(a, b); }); }
    __device__ __forceinline__ uint32_t min(uint32_t v) const { return reduce(v, [](uint32_t a, uint32_t b) { return a < b ? a : b; }); }
    __device__ __forceinline__ bool any(bool v) const { return reduce((int)v, [](int a, int b) { return a | b; }) != 0; }
    __device__ __forceinline__ double sum(double v) const {
        for (uint32_t o = lanes / 2; o; o >>= 1) v += __shfl_xor(v, o);
        return v;
    }
};
typedef PartOf<0> Part;

// The best two of two such pairs.
template <class C>
__device__ __forceinline__ void best_two(C& first, C& second, C a, C b) {
    const C low = first < a ? first : a;
    first = first < a ? a : first;
    second = second < b ? b : second;
    second = second < low ? low : second;
}

template <>
__device__ __forceinline__ void best_two<float>(float& first, float& second, float a, float b) {
    second = fmaxf(fmaxf(second, b), fminf(first, a));
    first = fmaxf(first, a);
}
// The best two of `lanes` lanes' two.
__device__ __forceinline__ void best_two_of(uint32_t lanes, float& first, float& second) {
    if (lanes > 1) best_two(first, second, Part::moved<0xb1>(first), Part::moved<0xb1>(second));
    if (lanes > 2) best_two(first, second, Part::moved<0x4e>(first), Part::moved<0x4e>(second));
    if (lanes > 4) best_two(first, second, Part::moved<0x141>(first), Part::moved<0x141>(second));
    if (lanes > 8) best_two(first, second, Part::moved<0x140>(first), Part::moved<0x140>(second));
    if (lanes > 16) best_two(first, second, __shfl_xor(first, 16), __shfl_xor(second, 16));
    if (lanes > 32) best_two(first, second, __shfl_xor(first, 32), __shfl_xor(second, 32));
}

// Groups of any size, by way of LDS (row: the token's c by expert, then the groups' values): what is not in one of the top groups becomes
// NONE in `row`.  *least, *next: the values of the last group that is in and of the first that is not.
template <class C, class P>
__device__ __forceinline__ void choose_groups(const RouteCall& r, const P& part, uint32_t lane, C* row, C* least, C* next) {
    constexpr C NONE = -(C)INFINITY;
    const uint32_t size = r.experts / r.groups;
    C* of_group = row + r.experts;
    for (uint32_t g = lane; g < r.groups; g += part.lanes) {
        C first = NONE, second = NONE;
        for (uint32_t e = 0; e < size; ++e) best_two(first, second, row[g * size + e], NONE);
        of_group[g] = r.group_top == 2 && second != NONE ? first + second : first;
    }
    lanes_exchange();
    *least = INFINITY;
    *next = NONE;
    for (uint32_t g = lane; g < r.groups; g += part.lanes) {
        const C y = of_group[g];
        uint32_t better = 0;
        for (uint32_t o = 0; o < r.groups; ++o) better += of_group[o] > y || (of_group[o] == y && o < g);
        const bool out = better >= r.top_groups;
        if (out || y == NONE)
            for (uint32_t e = 0; e < size; ++e) row[g * size + e] = NONE;
        if (out && y > *next) *next = y;
        if (!out && y < *least) *least = y;
    }
    lanes_exchange();
}

// A token in binary64, value by value in LDS.  SLOTS_BY_LOGIT: by scores only the groups (there is no bias).
template <int IN, bool SLOTS_BY_LOGIT>
__device__ __forceinline__ void route_in_binary64(const RouteCall& r, const Part& part, uint32_t lane, uint32_t i, double from, double* row, int32_t* slot) {
    constexpr double NONE = -INFINITY;
    double sum = 0.0;
    for (uint32_t e = lane; e < r.experts; e += part.lanes) {
        double x = (double)element<IN>(r.x, (int64_t)i * r.ld + e);
        if (x != x) x = NONE;
        const double s = r.sigmoid ? 1.0 / (1.0 + exp(-x)) : exp(x - from);
        row[e] = x == NONE ? NONE : s;
        if (x != NONE) sum += s;
    }
    sum = part.sum(sum);
    for (uint32_t e = lane; e < r.experts; e += part.lanes) {
        double s = row[e];
        if (s == NONE) continue;
        if (!r.sigmoid) s /= sum;
        if (!SLOTS_BY_LOGIT) s += (double)r.bias[e];
        row[e] = s != s ? NONE : s;
    }
    lanes_exchange();
    double least, next;
    if (r.top_groups < r.groups) choose_groups(r, part, lane, row, &least, &next);
    if (SLOTS_BY_LOGIT)
        for (uint32_t e = lane; e < r.experts; e += part.lanes) row[e] = row[e] == NONE ? NONE : (double)element<IN>(r.x, (int64_t)i * r.ld + e);
    for (uint32_t k = 0; k < r.slots; ++k) {
        double best = NONE;
        uint32_t at = 0xffffffffu;
        for (uint32_t e = lane; e < r.experts; e += part.lanes)
            if (row[e] > best) best = row[e], at = e;
        for (uint32_t o = part.lanes / 2; o; o >>= 1) {
            const double other = __shfl_xor(best, o);
            const uint32_t other_at = __shfl_xor(at, o);
            if (other > best || (other == best && other_at < at)) best = other, at = other_at;
        }
        lanes_exchange();
        if (lane == 0) {
            slot[k] = best == NONE ? -1 : (int32_t)at;
            if (best != NONE) row[at] = NONE;
        }
        lanes_exchange();
    }
}

// What binary32 may be off in c = s + bias, relative to 1 + the token's largest |c|.  e^d by way of 2^(d log2 e), two rounded factors and the function's
// last place: |d| 2^-23.4 + 2^-23 of it.
//   sigmoid  s (1 - s) of that (|x| s (1 - s) < 0.23), s (2^-24 + 2^-23) for the sum and the reciprocal, 2^-24 |c| for the bias: below 2^-22 (1 + |c|)
//   softmax  d = x - m is rounded too, |d| 2^-22.6: p |d| < 0.37 of its own, and p times the mean of |d| over the distribution, below 1.8 for 1024 experts,
//            for the sum; p 2^-21.4 for functions, quotient and product: below 2^-20.4 (1 + |c|)
constexpr float OFF_SIGMOID = 0x1p-22f, OFF_SOFTMAX = 0x1p-20f;

// At least `wanted` of a token's lanes have a largest c that is not below what this returns.
template <class P>
__device__ __forceinline__ float bound_of(const P& part, float best, uint32_t wanted) {
    uint32_t greater = 0;
    auto count = [&](float other) { greater += other > best; };
    if (part.lanes == 16) {
        count(Part::moved<0x121>(best)), count(Part::moved<0x122>(best)), count(Part::moved<0x123>(best)), count(Part::moved<0x124>(best));   // row_ror
        count(Part::moved<0x125>(best)), count(Part::moved<0x126>(best)), count(Part::moved<0x127>(best)), count(Part::moved<0x128>(best));
        count(Part::moved<0x129>(best)), count(Part::moved<0x12a>(best)), count(Part::moved<0x12b>(best)), count(Part::moved<0x12c>(best));
        count(Part::moved<0x12d>(best)), count(Part::moved<0x12e>(best)), count(Part::moved<0x12f>(best));
    } else {
        for (uint32_t o = 1; o < part.lanes; ++o) count(__shfl_xor(best, o));
    }
    return -part.max(greater < wanted ? -best : -INFINITY);
}

// The wavefront's LDS: candidates of its tokens, or their experts and groups, or one token's in binary64.
constexpr uint32_t CANDIDATES = 64;
struct Candidate {
    float c;
    uint32_t expert;
};

// What groups and slots go by.  Scores saturate where logits still differ (a sigmoid in binary64 is 1 from 37 on), so slots go by the logits unless a bias is
// added; two scores of a group are added as they are.
enum RouteBy { BY_LOGITS, GROUPS_BY_SCORE, ALL_BY_SCORE };

// lds: bytes of a wavefront besides its slots (and their c).
template <int IN, int CHUNKS, int LANES, RouteBy BY, bool GROUPS>
__global__ void __launch_bounds__(256) k_route(RouteCall r, uint32_t lds) {
    typedef TokenLanes<IN, CHUNKS> L;
    constexpr float NONE = -INFINITY;
    constexpr bool BY_SCORE = BY == ALL_BY_SCORE, SCORES = BY != BY_LOGITS;
    extern __shared__ __align__(16) char shared[];
    if (LANES) r.lanes = LANES;
    const L l(r.experts, r.lanes);
    const PartOf<LANES> part(r.lanes);
    const uint32_t wave = threadIdx.x >> 6, at_once = l.tokens(), tokens = (blockDim.x >> 6) * at_once;      // of the workgroup
    const uint32_t mine = wave * at_once + l.of, of_group = r.experts / r.groups;
    char* own = shared + wave * lds;
    int32_t* slot = reinterpret_cast<int32_t*>(shared + (blockDim.x >> 6) * lds) + mine * r.slots;
    float* in_order = reinterpret_cast<float*>(shared + (blockDim.x >> 6) * lds) + tokens * r.slots + mine * (r.slots + 1);      // (BY_SCORE) the slots' c and the next
    // groups that are whole runs of lanes: `per` of them
    const uint32_t per = of_group / L::WIDTH;           // (at least WIDTH experts each: no more groups than CHUNKS a lane)
    const bool by_lanes = GROUPS && of_group % L::WIDTH == 0 && (per & (per - 1)) == 0 && per <= r.lanes;
    const uint32_t per_shift = by_lanes ? 31 - __clz(per) : 0;
    const bool at_a_time = r.lanes >= 16 && r.slots < r.lanes;
    const uint32_t base = blockIdx.x * tokens;
    const uint32_t i = base + mine;
    const bool in = i < r.tokens && !(r.keep && !r.keep[i]);
    words4 raw[CHUNKS];
    if (in) {
        l.load(r.x, (int64_t)i * r.ld, raw);
    } else {
        constexpr uint32_t none = IN == OUT_F32 ? 0xff800000u : IN == OUT_BF16 ? 0xff80ff80u : 0xfc00fc00u;
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) raw[k] = words4{none, none, none, none};
    }
    float c[L::N];
    L::unpack(raw, c);
    bool nan = false;
#pragma unroll
    for (int v = 0; v < L::N; v += 2) nan |= __builtin_isunordered(c[v], c[v + 1]);
    if (__any(nan)) {
#pragma unroll
        for (int v = 0; v < L::N; ++v) c[v] = c[v] != c[v] ? NONE : c[v];
    }
    float m = NONE;
#pragma unroll
    for (int v = 0; v < L::N; ++v) {
        c[v] = __builtin_canonicalizef(c[v]);                                       // known to be no signalling NaN, which costs maxima nothing then
        m = fmaxf(m, c[v]);
    }
    m = part.max(m);
    nan = part.any(nan) || (!r.sigmoid && m == INFINITY);
    const float from = m == NONE ? 0.0f : m;
    float by = 1.0f;                                                            // softmax: 1 / sum of e^(x - m)
    bool close = false;
    float off = 0.0f;
    if (SCORES) {
        if (!r.sigmoid) {
            double sum = 0.0;
#pragma unroll
            for (int v = 0; v < L::N; ++v) sum += (double)exp_of(c[v] - from);
            by = (float)(1.0 / part.sum(sum));
        }
        float bias[L::N];
#pragma unroll
        for (int v = 0; v < L::N; ++v) bias[v] = 0.0f;
        if (BY_SCORE && r.bias) {         // always there: without the branch its loads go out early and hold registers (131072 x 256: 80 us, with it 76)
#pragma unroll
            for (int v = 0; v < L::N; v += 4) {
                if (l.expert(v) + 4 <= r.experts) {
                    const words4 four = *reinterpret_cast<const words4*>(r.bias + l.expert(v));
#pragma unroll
                    for (int e = 0; e < 4; ++e) bias[v + e] = __uint_as_float(four[e]);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (l.expert(v) + e < r.experts) bias[v + e] = r.bias[l.expert(v) + e];
                }
            }
        }
#pragma unroll
        for (int v = 0; v < L::N; ++v) {
            const float s = (r.sigmoid ? __builtin_amdgcn_rcpf(1.0f + exp_of(-c[v])) : exp_of(c[v] - from) * by) + bias[v];
            c[v] = ((c[v] == NONE) | (s != s)) ? NONE : s;
            off = fmaxf(off, c[v] == NONE ? 0.0f : fabsf(c[v]));
        }
        off = (r.sigmoid ? OFF_SIGMOID : OFF_SOFTMAX) * (1.0f + part.max(off));
    } else if (!r.sigmoid && !r.renormalise) {
        float sum = 0.0f;
#pragma unroll
        for (int v = 0; v < L::N; ++v) sum += expf(c[v] - from);
        by = 1.0f / part.sum(sum);
    }
    if (GROUPS) {
        float least, next;
        if (by_lanes) {
            float* values = reinterpret_cast<float*>(own) + l.of * r.groups;
#pragma unroll
            for (int k = 0; k < CHUNKS; ++k) {
                float first = NONE, second = NONE;
#pragma unroll
                for (int w = 0; w < L::WIDTH; ++w) best_two(first, second, c[k * L::WIDTH + w], NONE);
                best_two_of(per, first, second);
                const uint32_t g = (k * r.lanes + l.lane) >> per_shift;
                if (g < r.groups) values[g] = r.group_top == 2 && second != NONE ? first + second : first;
            }
            lanes_exchange();
            least = INFINITY;
            next = NONE;
            uint64_t out = 0;                                                       // of this lane's groups: as many as it has chunks at most
            for (uint32_t g = l.lane, j = 0; g < r.groups; g += r.lanes, ++j) {
                const float y = values[g];
                uint32_t better = 0;
#pragma unroll 4
                for (uint32_t o = 0; o < r.groups; ++o) {
                    const float other = values[o];
                    better += (other > y) | ((other == y) & (o < g));
                }
                if (better < r.top_groups) {
                    least = fminf(least, y);
                } else {
                    next = fmaxf(next, y);
                    out |= 1ull << j;
                }
            }
            lanes_exchange();
            for (uint32_t g = l.lane, j = 0; g < r.groups; g += r.lanes, ++j)
                if (out >> j & 1) values[g] = NAN;
            lanes_exchange();
#pragma unroll
            for (int k = 0; k < CHUNKS; ++k) {
                const uint32_t g = (k * r.lanes + l.lane) >> per_shift;
                const float y = values[min(g, r.groups - 1)];
#pragma unroll
                for (int w = 0; w < L::WIDTH; ++w) c[k * L::WIDTH + w] = y != y ? NONE : c[k * L::WIDTH + w];
            }
        } else {
            float* row = reinterpret_cast<float*>(own) + l.of * (r.experts + r.groups);
#pragma unroll
            for (int v = 0; v < L::N; ++v)
                if (l.expert(v) < r.experts) row[l.expert(v)] = c[v];
            lanes_exchange();
            choose_groups(r, part, l.lane, row, &least, &next);
#pragma unroll
            for (int v = 0; v < L::N; ++v) c[v] = l.expert(v) < r.experts ? row[l.expert(v)] : NONE;
        }
        lanes_exchange();
        if (SCORES) {
            least = -part.max(-least);
            next = part.max(next);
            close |= least != NONE && !(least - next > 4.0f * off);             // sums of two, each off; infinities are close
        }
        if (BY == GROUPS_BY_SCORE) {
            float x[L::N];
            L::unpack(raw, x);
#pragma unroll
            for (int v = 0; v < L::N; ++v) c[v] = c[v] == NONE ? NONE : __builtin_canonicalizef(x[v]);
        }
    }
    // All slots at once: the slots' lanes' largest c bound what can be chosen, and few c are not below that; each of those finds its
    // place by comparing with the others.  (With a score one more than the slots, which must not be close to the last.)
    constexpr uint32_t MORE = BY_SCORE ? 1 : 0;
    bool done = false;
    if (at_a_time) {
        float best = NONE;
#pragma unroll
        for (int v = 0; v < L::N; ++v) best = fmaxf(best, c[v]);
        const float bound = fmaxf(bound_of(part, best, r.slots + MORE), -3.4028235e38f);
        uint32_t count = 0;
#pragma unroll
        for (int v = 0; v < L::N; ++v) count += c[v] >= bound;
        uint32_t to = count;
        for (uint32_t o = 1; o < r.lanes; o <<= 1) {
            const uint32_t other = __shfl_up(to, o);
            if (l.lane >= o) to += other;
        }
        const uint32_t n = __shfl(to, (threadIdx.x & 63) | (r.lanes - 1));
        to -= count;
        done = !__any(n > CANDIDATES);
        if (done) {
            Candidate* list = reinterpret_cast<Candidate*>(own) + l.of * CANDIDATES;
#pragma unroll
            for (int v = 0; v < L::N; ++v)
                if (c[v] >= bound) list[to++] = Candidate{c[v], l.expert(v)};
            for (uint32_t k = l.lane; k < r.slots + MORE; k += r.lanes) {
                if (k < r.slots) slot[k] = -1;
                if (BY_SCORE) in_order[k] = NONE;
            }
            lanes_exchange();
            for (uint32_t k = l.lane; k < n; k += r.lanes) {
                const Candidate me = list[k];
                uint32_t before = 0;
                for (uint32_t o = 0; o < n; ++o) {
                    const Candidate other = list[o];
                    before += (other.c > me.c) | ((other.c == me.c) & (other.expert < me.expert));
                }
                if (before < r.slots) slot[before] = (int32_t)me.expert;
                if (BY_SCORE && before <= r.slots) in_order[before] = me.c;
            }
            lanes_exchange();
            if (BY_SCORE) {
                for (uint32_t k = l.lane; k < r.slots; k += r.lanes) close |= in_order[k + 1] != NONE && !(in_order[k] - in_order[k + 1] > 2.0f * off);
                close = part.any(close);
            }
        }
    }
    if (!done) {                        // of equal c the lower expert, which is also the lower v of a lane
        float before = INFINITY;
        for (uint32_t k = 0; k < r.slots + MORE; ++k) {
            float best = NONE;
#pragma unroll
            for (int v = 0; v < L::N; ++v) best = fmaxf(best, c[v]);
            best = part.max(best);
            if (BY_SCORE) {
                close |= k && best != NONE && !(before - best > 2.0f * off);
                before = best;
                if (k == r.slots) break;
            }
            uint32_t at = 0xffffffffu;
#pragma unroll
            for (int v = L::N; v-- > 0;) at = c[v] == best ? l.expert(v) : at;
            at = part.min(at);
#pragma unroll
            for (int v = 0; v < L::N; ++v) c[v] = l.expert(v) == at ? NONE : c[v];
            if (l.lane == 0) slot[k] = best == NONE ? -1 : (int32_t)at;
        }
        lanes_exchange();
    }
    if (SCORES) {
        for (uint64_t again = __ballot(close && in && l.lane == 0); again; again &= again - 1) {
            const uint32_t lane = __ffsll((unsigned long long)again) - 1, token = wave * at_once + lane / r.lanes;
            route_in_binary64<IN, !BY_SCORE>(r, Part(64), threadIdx.x & 63, base + token, (double)__shfl(from, lane), reinterpret_cast<double*>(own),
                                  slot + ((int32_t)token - (int32_t)mine) * (int32_t)r.slots);
        }
    }
    if (i < r.tokens) {
        // a lane's slots: the first's logit is at hand, more than one are read again
        auto logit = [&](int32_t e) { return element<IN>(r.x, (int64_t)i * r.ld + e); };
        const int32_t mine0 = l.lane < r.slots ? slot[l.lane] : -1;
        const float x0 = mine0 >= 0 ? logit(mine0) : NONE;
        auto share = [&](float x, float m) { return r.sigmoid ? sigmoid_over(x, m) : expf(x - m); };
        float all = 1.0f, most = r.sigmoid ? 0.0f : m, q0 = 0.0f;
        if (r.renormalise) {
            most = r.sigmoid && mine0 >= 0 ? fminf(x0, 0.0f) : x0;
            for (uint32_t k = l.lane + r.lanes; k < r.slots; k += r.lanes)
                if (slot[k] >= 0) most = fmaxf(most, r.sigmoid ? fminf(logit(slot[k]), 0.0f) : logit(slot[k]));
            most = part.max(most);
            q0 = mine0 >= 0 ? share(x0, most) : 0.0f;
            all = q0;
            for (uint32_t k = l.lane + r.lanes; k < r.slots; k += r.lanes)
                if (slot[k] >= 0) all += share(logit(slot[k]), most);
            all = part.sum(all);
        } else if (mine0 >= 0) {
            q0 = share(x0, most);
        }
        for (uint32_t k = l.lane; k < r.slots; k += r.lanes) {
            const int32_t e = slot[k];
            float y = 0.0f;
            if (e >= 0) y = (k == l.lane ? q0 : share(logit(e), most)) * (r.renormalise || r.sigmoid ? 1.0f : by) / all * r.scale;
            const size_t to = (size_t)i * r.slots + k;
            r.chosen[to] = e;
            r.weight[to] = nan ? NAN : y;
        }
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

template <int IN, int CHUNKS>
__global__ void __launch_bounds__(256) k_route_gradient(RouteGradient r) {
    typedef TokenLanes<IN, CHUNKS> L;
    extern __shared__ __align__(16) char shared[];
    const L l(r.experts, r.lanes);
    const Part part(r.lanes);
    const uint32_t wave = threadIdx.x >> 6, at_once = l.tokens(), tokens = (blockDim.x >> 6) * at_once;
    const uint32_t mine = wave * at_once + l.of;
    const uint32_t units = (r.experts + L::WIDTH - 1) / L::WIDTH * L::WIDTH;
    f32_bytes* row = reinterpret_cast<f32_bytes*>(shared) + (size_t)mine * units;
    SlotGradient* slot = reinterpret_cast<SlotGradient*>(shared + (size_t)tokens * units * sizeof(float)) + (size_t)mine * r.slots;
    const bool dense = !r.sigmoid && !r.renormalise;
    const uint32_t i = blockIdx.x * tokens + mine;
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
    // by expert: the slots' parts in their order, so that the sum of an expert's is the same every time
#pragma unroll
    for (int v = 0; v < L::N; v += 4)
        if (l.expert(v) < units) *reinterpret_cast<f32x4_bytes*>(row + l.expert(v)) = f32x4{};
    lanes_exchange();
    for (uint32_t k = l.lane; k < r.slots; k += r.lanes) {
        const SlotGradient s = slot[k];
        if (s.expert >= r.experts) continue;
        bool first = true;
        float sum = s.d;
        for (uint32_t o = 0; o < r.slots; ++o) {
            if (o == k || slot[o].expert != s.expert) continue;
            first &= o > k;
            sum += slot[o].d;
        }
        if (first) row[s.expert] = sum;
    }
    lanes_exchange();
    float d[L::N];
#pragma unroll
    for (int v = 0; v < L::N; v += 4) {
        f32x4 four = {};
        if (l.expert(v) < units) four = *reinterpret_cast<const f32x4_bytes*>(row + l.expert(v));
#pragma unroll
        for (int e = 0; e < 4; ++e) d[v + e] = four[e];
    }
    if (i >= r.tokens) return;
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

}  // namespace iwp
