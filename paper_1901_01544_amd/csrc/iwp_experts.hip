// Host side of the C ABI declared in include/iwp_experts.h: argument checks, workspace carving and launch sequences.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "iwp_host.hpp"
#include "iwp_route.hpp"

using namespace iwp;

namespace {

inline bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
inline size_t size_of(uint32_t dtype) { return dtype == IWP_F32 ? 4 : 2; }

// f(lanes of a token, constant with the chunks of 16 bytes of a lane): 16 bytes a lane up to 16 lanes, then two and four times as many.
template <int IN, class F>
int with_lanes(uint32_t experts, F f) {
    const uint32_t units = (experts + TokenLanes<IN, 1>::WIDTH - 1) / TokenLanes<IN, 1>::WIDTH;
    const uint32_t chunks = units <= 16 ? 1 : units <= 32 ? 2 : 4;
    uint32_t lanes = 1;
    while (lanes * chunks < units) lanes *= 2;
    if (chunks == 1) return f(lanes, std::integral_constant<int, 1>{});
    return chunks == 2 ? f(lanes, std::integral_constant<int, 2>{}) : f(lanes, std::integral_constant<int, 4>{});
}

template <class F>
int with_type(uint32_t dtype, F f) {
    if (dtype == IWP_F32) return f(std::integral_constant<int, OUT_F32>{});
    return dtype == IWP_BF16 ? f(std::integral_constant<int, OUT_BF16>{}) : f(std::integral_constant<int, OUT_F16>{});
}

constexpr uint32_t LDS_OF_A_LAUNCH = 65536;
constexpr uint32_t ROUTE_GROUPS = 4096;

// Launches over tokens: wavefronts of a workgroup (as many of four as LDS has room for) and workgroups.
struct TokenGrid {
    uint32_t waves = 4, lds, blocks;
    TokenGrid(uint32_t tokens, uint32_t lanes, uint32_t bytes_per_token) {
        const uint32_t at_once = 64 / lanes;
        while (waves > 1 && waves * at_once * bytes_per_token > LDS_OF_A_LAUNCH) waves /= 2;
        lds = waves * at_once * bytes_per_token;
        blocks = std::min((tokens + waves * at_once - 1) / (waves * at_once), ROUTE_GROUPS);
    }
};

}  // namespace

extern "C" {

int iwp_route(const void* x, int64_t ld_x, uint32_t tokens, uint32_t experts, uint32_t dtype, const float* bias, uint32_t scores,
              uint32_t groups, uint32_t top_groups, uint32_t group_top, uint32_t renormalise, float scale, const uint8_t* keep,
              int32_t* chosen, float* weight, uint32_t slots, void* hip_stream) {
    if (tokens > IWP_MAX_TOKENS || experts < 1 || experts > IWP_MAX_EXPERTS || dtype > IWP_F16 || scores > IWP_SIGMOID || renormalise > 1)
        return IWP_EINVAL;
    if (groups < 1 || experts % groups || top_groups < 1 || top_groups > groups || group_top < 1 || group_top > 2 || group_top > experts / groups)
        return IWP_EINVAL;
    if (slots < 1 || slots > top_groups * (experts / groups) || !std::isfinite(scale) || ld_x < experts) return IWP_EINVAL;
    if (tokens && (!x || !chosen || !weight)) return IWP_EINVAL;
    if (!aligned(x, size_of(dtype)) || !aligned(bias, 4) || !aligned(chosen, 4) || !aligned(weight, 4)) return IWP_EALIGN;
    if (tokens == 0) return IWP_OK;
    const hipStream_t s = static_cast<hipStream_t>(hip_stream);
    const bool grouped = top_groups < groups, by_score = bias || (grouped && group_top == 2);
    return with_type(dtype, [&](auto in) {
        return with_lanes<in.value>(experts, [&](uint32_t lanes, auto chunks) {
            constexpr int IN = decltype(in)::value, CHUNKS = decltype(chunks)::value;
            const RouteCall r{x, ld_x, tokens, experts, lanes, slots, bias, scores == IWP_SIGMOID, renormalise != 0, groups, top_groups, group_top,
                              scale, keep, chosen, weight};
            const TokenGrid g(tokens, lanes, (uint32_t)(slots * sizeof(Slot) + (grouped ? (experts + groups) * (by_score ? 8 : 4) : 0)));
            auto launch = [&](auto kernel) {
                IWP_LAUNCH_AS("k_route", kernel, g.blocks, g.waves * 64, g.lds, s, r);
                return (int)IWP_OK;
            };
            if (by_score) return grouped ? launch(k_route<IN, CHUNKS, double, true>) : launch(k_route<IN, CHUNKS, double, false>);
            return grouped ? launch(k_route<IN, CHUNKS, float, true>) : launch(k_route<IN, CHUNKS, float, false>);
        });
    });
}

int iwp_route_gradient(const void* x, int64_t ld_x, uint32_t tokens, uint32_t experts, uint32_t dtype, const int32_t* chosen,
                       const float* dweight, uint32_t slots, uint32_t scores, uint32_t renormalise, float scale, const uint8_t* keep,
                       const void* plus, int64_t ld_plus, void* dx, int64_t ld_dx, void* hip_stream) {
    if (tokens > IWP_MAX_TOKENS || experts < 1 || experts > IWP_MAX_EXPERTS || dtype > IWP_F16 || scores > IWP_SIGMOID || renormalise > 1)
        return IWP_EINVAL;
    if (slots < 1 || slots > experts || !std::isfinite(scale) || ld_x < experts || ld_dx < experts || (plus && ld_plus < experts)) return IWP_EINVAL;
    if (tokens && (!x || !chosen || !dweight || !dx)) return IWP_EINVAL;
    const size_t e = size_of(dtype);
    if (!aligned(x, e) || !aligned(plus, e) || !aligned(dx, e) || !aligned(chosen, 4) || !aligned(dweight, 4)) return IWP_EALIGN;
    if (tokens == 0) return IWP_OK;
    const hipStream_t s = static_cast<hipStream_t>(hip_stream);
    return with_type(dtype, [&](auto in) {
        return with_lanes<in.value>(experts, [&](uint32_t lanes, auto chunks) {
            constexpr int IN = decltype(in)::value, CHUNKS = decltype(chunks)::value;
            const RouteGradient r{x, ld_x, tokens, experts, lanes, slots, chosen, dweight, scores == IWP_SIGMOID, renormalise != 0, scale, keep,
                                  plus, ld_plus, dx, ld_dx};
            const TokenGrid g(tokens, lanes, (uint32_t)(slots * sizeof(SlotGradient)));
            auto kernel = k_route_gradient<IN, CHUNKS>;
            IWP_LAUNCH_AS("k_route_gradient", kernel, g.blocks, g.waves * 64, g.lds, s, r);
            return (int)IWP_OK;
        });
    });
}

}  // extern "C"
