// Host side of the C ABI declared in include/iwp_experts.h: argument checks, workspace carving and launch sequences.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "iwp_grouped.hpp"
#include "iwp_host.hpp"
#include "iwp_launch_rows.hpp"
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

// Launches over tokens: wavefronts of a workgroup (as many of four as LDS has room for) and workgroups.
struct TokenGrid {
    uint32_t waves = 4, lds, blocks;
    TokenGrid(uint32_t tokens, uint32_t at_once, uint32_t bytes_per_wave) {
        while (waves > 1 && waves * bytes_per_wave > LDS_OF_A_LAUNCH) waves /= 2;
        lds = waves * bytes_per_wave;
        blocks = (tokens + waves * at_once - 1) / (waves * at_once);
    }
};

template <class T>
T round_up(T x, T to) { return (x + to - 1) / to * to; }

// ------------------------------------------------------------------ the products

struct Big { static constexpr int BP = 256, BQ = 256, WP = 2, WQ = 4, THREADS = 512; };
struct Mid { static constexpr int BP = 128, BQ = 128, WP = 2, WQ = 2, THREADS = 256; };
struct Few { static constexpr int BP = 64, BQ = 64, WP = 2, WQ = 2, THREADS = 256; };
enum TileKind { BIG, MID, FEW };

template <class F>
int with_tile(TileKind kind, F f) {
    switch (kind) {
        case BIG: return f(Big{});
        case MID: return f(Mid{});
        default: return f(Few{});
    }
}

// Of a kind of operands: binary32 takes the small tiles alone.
template <class K, class F>
int with_tile_of(TileKind kind, F f) {
    if constexpr (K::OUT == OUT_F32) return f(Few{});
    else return with_tile(kind, f);
}

template <class T>
uint64_t tiles_of(uint64_t np, uint64_t nq) { return (np + T::BP - 1) / T::BP * ((nq + T::BQ - 1) / T::BQ); }

// The largest tile of which the experts' rows make enough for most of the 256 compute units and that they fill.  us of a call with large tiles, middling
// and small ones, bf16: 2048 x 2 rows of 8 experts x 2048 x 4096 (512 rows each) 119, 111, 130; 8192 x 8 of 32 x 1024 x 512 (2048 each) 145, 141, 164; 512 x 2
// of 8 x 2048 x 4096 (128 each) 58, 44, 55; 64 x 4 of 16 x 2048 x 2048 (16 each) 52, 36, 31.  Binary32 is bound by the matrix cores in any tile and
// wants them small: 4096 x 2 of 8 x 1024 x 1024 272, 288, 183.
constexpr uint64_t ENOUGH_TILES = 160;
// `each`: entries of Q that one expert has; `many`: experts that have that many
TileKind tile_for(uint64_t np, uint64_t each, uint64_t many, uint32_t dtype) {
    if (dtype == IWP_F32) return FEW;
    if (many * tiles_of<Big>(np, each) >= ENOUGH_TILES && each > Mid::BQ) return BIG;
    return many * tiles_of<Mid>(np, each) >= ENOUGH_TILES && each > Few::BQ ? MID : FEW;
}

struct Carver {            // hands out 256-byte aligned parts; at == nullptr: only adds up
    char* at;
    size_t used = 0;
    template <class T>
    void take(T*& p, size_t n) {
        p = at ? reinterpret_cast<T*>(at + used) : nullptr;
        used += (n * sizeof(T) + 255) & ~size_t(255);
    }
};

struct ProductSizes {
    uint32_t tokens, slots, experts, in, out, dtype;
    bool by_slot, gradient;
    uint32_t rows() const { return tokens * slots; }
    // rows of the gathered matrices: those of an expert end at a multiple of PAD_ROWS
    uint32_t padded() const { return rows() + std::min(experts, rows()) * (PAD_ROWS - 1); }
    bool ok() const {
        return tokens <= IWP_MAX_TOKENS && slots >= 1 && experts >= 1 && experts <= IWP_MAX_EXPERTS && slots <= experts &&
               (uint64_t)tokens * slots <= IWP_MAX_ROWS && in >= 1 && in <= IWP_MAX_DIM && out >= 1 && out <= IWP_MAX_DIM && dtype <= IWP_F16;
    }
};

struct ProductPlan {
    uint32_t deep, ld_x, ld_d;             // elements in 128 bytes; widths rounded up to that
    TileKind tile;
    uint32_t height, max_tiles;
    uint32_t arrangers, per_wave;          // workgroups that arrange the slots, slots of a wavefront
    ExpertRows R;
    char *x, *d, *w;                       // gathered rows, gathered gradients, copied matrices
    float* sums;
    size_t bytes;
};

bool readable(const void* w, int64_t ld, int64_t step, uint32_t in, uint32_t dtype) {
    const int64_t chunk = 16 / size_of(dtype);
    return aligned(w, 16) && ld % chunk == 0 && step % chunk == 0 && in % chunk == 0;
}

// Matrices that the tiles cannot load by 16 bytes a lane are copied to rows of whole units first, except for binary32's, whose entries are a load's
// least width: there tiles load them by 4 bytes.  us of a call with the copy and without: 2050 rows of 17 x 1001 x 777 85 and 68; both gradients of 256 rows
// of 16 x 2047 x 2048 354 and 260.
bool copies_matrices(const void* w, int64_t ld, int64_t step, uint32_t in, uint32_t dtype) { return dtype != IWP_F32 && !readable(w, ld, step, in, dtype); }
// f(constant with the bytes of a matrix that a lane loads)
template <class K, class F>
int with_lane(bool by_chunks, F f) {
    if constexpr (K::OUT == OUT_F32)
        if (!by_chunks) return f(std::integral_constant<int, 4>{});
    return f(std::integral_constant<int, 16>{});
}

// One workgroup arranges up to 2048 slots; more are counted first and arranged by up to 64, each of which reads all the others' counts, 1024
// slots or more each.  us of counting and arranging: 2042 slots by one 10, by two 16; 4096 by one 13, by four 16 (a call with small products 14.5 and
// 13.8); 16384 of 8 experts by 4 21, by 16 17.  Beside a copy of the matrices, which takes longer, one workgroup is enough for more.
constexpr uint32_t ARRANGE_ONE = 2048, ARRANGE_SLOTS = 1024, ARRANGE_MOST = 64;

// Products of few rows an expert need no arrangement.  us here and by tiles, mean rows of an expert that has any: bf16 1 token x 8 of 64 experts x 2048 x 1024
// 10 and 33, 16 tokens 42 and 53 (2 rows), 32 x 4 of 16 x 2048 x 2048 34 and 42 (8), 64 x 4 of 16 50 and 42 (16); binary32 60 x 2 of 8 x 1024 x 1024
// 16 and 29 (15).  The host knows no more than the mean.  Where all rows are one expert's, its matrix is read again for every 16 of them by the few
// workgroups that it has: 512 rows of 64 x 2048 x 1024 in bf16 126 (evenly 57; 520 rows, by tiles, 28 and 48), 128 rows 33 (40), 32 rows 10 (20); 1024 rows of
// 64 x 1024 x 1024 in binary32 258 (90; 1025 rows, by tiles, 49 and 85).
bool few_rows(const ProductSizes& z) {
    const uint32_t n = z.rows();
    return n <= FEW_SLOTS && n <= (z.dtype == IWP_F32 ? FEW_ROWS : FEW_ROWS / 2) * std::min(z.experts, n);
}

ProductPlan product_plan(const ProductSizes& z, bool copy_w, void* workspace) {
    ProductPlan p{};
    p.deep = ROW_BYTES / (uint32_t)size_of(z.dtype);
    p.ld_x = round_up(z.in, p.deep);
    p.ld_d = round_up(z.out, p.deep);
    const uint32_t n = z.rows(), many = std::max(1u, std::min(z.experts, n)), each = (n + many - 1) / many;
    p.tile = tile_for(z.gradient ? z.in : z.out, each, many, z.dtype);
    p.height = p.tile == BIG ? Big::BQ : p.tile == MID ? Mid::BQ : Few::BQ;
    p.max_tiles = n / p.height + many + 1;
    p.arrangers = n <= (copy_w ? 4 * ARRANGE_ONE : ARRANGE_ONE) ? 1 : std::min((n + ARRANGE_SLOTS - 1) / ARRANGE_SLOTS, ARRANGE_MOST);
    p.per_wave = round_up((n + p.arrangers * ARRANGE_WAVES - 1) / (p.arrangers * ARRANGE_WAVES), 64u);
    if (!z.gradient && few_rows(z)) {
        p.bytes = 256;                     // none is used
        return p;
    }
    Carver c{static_cast<char*>(workspace)};
    if (p.arrangers > 1) c.take(p.R.counts, (size_t)p.arrangers * (z.experts + 1));
    c.take(p.R.start, z.experts + 1);
    c.take(p.R.count, z.experts + 1);
    c.take(p.R.slot, (size_t)z.padded() + n);
    c.take(p.R.tile, p.max_tiles);
    c.take(p.R.tiles, 2);
    const size_t size = size_of(z.dtype);
    c.take(p.x, (size_t)z.padded() * p.ld_x * size);
    if (z.gradient) {
        c.take(p.d, (size_t)z.padded() * p.ld_d * size);
        if (!z.by_slot && z.slots > 1) c.take(p.sums, (size_t)n * p.ld_x);
    }
    if (copy_w) c.take(p.w, (size_t)z.experts * z.out * p.ld_x * size);
    p.bytes = c.used;
    return p;
}

Spread spread(uint32_t units) {
    Spread s{0, 1};
    while (s.shift < 8 && (1u << s.shift) < units) ++s.shift;
    s.across = (units + (1u << s.shift) - 1) >> s.shift;
    return s;
}

struct KindF32 { typedef F32 E; typedef FewF32 FEW_E; static constexpr int OUT = OUT_F32; };
struct KindBf16 { typedef Bf16 E; typedef FewBf16 FEW_E; static constexpr int OUT = OUT_BF16; };
struct KindF16 { typedef F16 E; typedef FewF16 FEW_E; static constexpr int OUT = OUT_F16; };

template <class F>
int with_kind(uint32_t dtype, F f) {
    if (dtype == IWP_F32) return f(KindF32{});
    return dtype == IWP_BF16 ? f(KindBf16{}) : f(KindF16{});
}

// Arranges the slots, and copies the matrices (if they are wanted and cannot be read where they lie) and `rows`.
template <int SIZE>
int arrange(const ProductSizes& z, const ProductPlan& p, const int32_t* chosen, const void* w, int64_t ld, int64_t step, bool wanted, Matrices* W,
            const MatrixCopy& rows, hipStream_t s) {
    *W = Matrices{static_cast<const char*>(w), step, (uint32_t)ld, z.out, z.in};
    MatrixCopy copy{static_cast<const char*>(w), ld, step, z.out, z.in, Units{1, 0}, p.w};
    if (p.w && wanted) {
        *W = Matrices{p.w, (int64_t)z.out * p.ld_x, p.ld_x, z.out, z.in};
        copy.of = Units{p.ld_x * SIZE / 16, z.experts * z.out};
    }
    const uint32_t copiers = (uint32_t)((copy.of.threads() + rows.of.threads() + ARRANGE_THREADS - 1) / ARRANGE_THREADS);
    if (p.arrangers > 1) IWP_LAUNCH_BLOCK("k_expert_count", k_expert_count, p.arrangers, ARRANGE_THREADS, s, chosen, z.rows(), p.per_wave, z.experts, p.R);
    IWP_LAUNCH_BLOCK("k_expert_arrange", k_expert_arrange<SIZE>, p.arrangers + copiers, ARRANGE_THREADS, s, chosen, z.rows(), p.per_wave, z.experts, p.height,
                     p.arrangers, p.R, copy, rows);
    return IWP_OK;
}

RowsGather gather_of(const ProductSizes& z, const void* x, int64_t ld, uint32_t dim, uint32_t slots, char* out, uint32_t ld_out) {
    return RowsGather{static_cast<const char*>(x), ld, dim, slots, Units{(uint32_t)(ld_out * size_of(z.dtype) / 16), z.padded()}, out};
}
template <int SIZE>
int gather(const ProductSizes& z, const ProductPlan& p, const RowsGather& A, const RowsGather& B, hipStream_t s) {
    const uint32_t a = (uint32_t)((A.of.threads() + 255) / 256), b = (uint32_t)((B.of.threads() + 255) / 256);
    if (a + b) IWP_LAUNCH_BLOCK("k_expert_gather", k_expert_gather<SIZE>, a + b, 256, s, A, B, a, z.experts, p.R);
    return IWP_OK;
}

// HIP counts a launch's threads in 32 bits.  More rows by columns than this allows fit no memory.
bool launches_fit(const ProductSizes& z, const ProductPlan& p) {
    const uint64_t widest = round_up(std::max(z.in, z.out), 64u), units = widest * size_of(z.dtype) / 16;
    return 2 * units * (z.padded() / GATHER_ROWS + 1) <= MOST_THREADS &&
           units * ((uint64_t)z.experts * z.out / GATHER_ROWS + z.rows() / GATHER_ROWS + 2) + (ARRANGE_MOST + 2) * ARRANGE_THREADS <= MOST_THREADS &&
           with_tile(p.tile, [&](auto tile) {
               typedef decltype(tile) T;
               const uint64_t rows = (widest + T::BP - 1) / T::BP * p.max_tiles, matrices = z.gradient ? z.experts * tiles_of<T>(z.in, z.out) : 0;
               return (int)((rows + matrices + TILES_AT_A_TIME) * T::THREADS <= MOST_THREADS);
           });
}

// Can a product read these rows where they lie?  By 16 bytes, whole tiles of the summed index, within what 32 bits count.
bool in_place(const void* x, int64_t ld, uint32_t dim, uint64_t rows, uint32_t dtype) {
    const uint64_t size = size_of(dtype);
    return aligned(x, 16) && ld * size % 16 == 0 && dim * size % ROW_BYTES == 0 && rows * ld * size < (uint64_t)1 << 32;
}

// What both calls check: sizes, x, w and chosen.
int product_checks(const ProductSizes& z, uint32_t x_by_slot, const void* x, int64_t ld_x, const void* w, int64_t ld_w, int64_t step_w, const int32_t* chosen) {
    if (!z.ok() || x_by_slot > 1 || !launches_fit(z, product_plan(z, false, nullptr))) return IWP_EINVAL;
    if (z.tokens && (!x || !chosen)) return IWP_EINVAL;
    if (!w || ld_x < z.in || ld_w < z.in || (z.experts > 1 && step_w < (int64_t)(z.out - 1) * ld_w + z.in)) return IWP_EINVAL;
    return IWP_OK;
}
bool too_far(int64_t ld, uint32_t dtype) { return ld >= (int64_t)((1u << 24) / size_of(dtype)); }

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
    const bool grouped = top_groups < groups, scored = bias || (grouped && group_top == 2);
    return with_type(dtype, [&](auto in) {
        return with_lanes<in.value>(experts, [&](uint32_t lanes, auto chunks) {
            constexpr int IN = decltype(in)::value, CHUNKS = decltype(chunks)::value;
            const RouteCall r{x, ld_x, tokens, experts, lanes, slots, bias, scores == IWP_SIGMOID, renormalise != 0, groups, top_groups, group_top,
                              scale, keep, chosen, weight};
            const uint32_t at_once = 64 / lanes, row = experts + groups;
            const uint32_t lds = round_up<uint32_t>(std::max({lanes >= 16 ? at_once * CANDIDATES * (uint32_t)sizeof(Candidate) : 0u, scored ? row * 8 : 0u,
                                                              grouped ? at_once * row * 4 : 0u}), 16);
            const TokenGrid g(tokens, at_once, lds + at_once * (bias ? 2 * slots + 1 : slots) * 4);
            auto launch = [&](auto kernel) {
                IWP_LAUNCH_AS("k_route", kernel, g.blocks, g.waves * 64, g.lds, s, r, lds);
                return (int)IWP_OK;
            };
            auto of_lanes = [&](auto known) {
                constexpr int LANES = decltype(known)::value;
                if (bias) return grouped ? launch(k_route<IN, CHUNKS, LANES, ALL_BY_SCORE, true>) : launch(k_route<IN, CHUNKS, LANES, ALL_BY_SCORE, false>);
                if (scored) return launch(k_route<IN, CHUNKS, LANES, GROUPS_BY_SCORE, true>);
                return grouped ? launch(k_route<IN, CHUNKS, LANES, BY_LOGITS, true>) : launch(k_route<IN, CHUNKS, LANES, BY_LOGITS, false>);
            };
            if (CHUNKS == 2 || lanes == 16) return of_lanes(std::integral_constant<int, 16>{});
            return of_lanes(std::integral_constant<int, CHUNKS == 2 ? 16 : 0>{});
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
            const uint32_t at_once = 64 / lanes;
            const TokenGrid g(tokens, at_once, at_once * (uint32_t)(slots * sizeof(SlotGradient) + (experts + 7) / 8 * 8 * sizeof(float)));
            auto kernel = k_route_gradient<IN, CHUNKS>;
            IWP_LAUNCH_AS("k_route_gradient", kernel, g.blocks, g.waves * 64, g.lds, s, r);
            return (int)IWP_OK;
        });
    });
}

size_t iwp_expert_product_workspace_bytes(uint32_t tokens, uint32_t slots, uint32_t experts, uint32_t in, uint32_t out, uint32_t dtype, const void* w,
                                          int64_t ld_w, int64_t step_w, uint32_t x_by_slot, uint32_t gradient) {
    const ProductSizes z{tokens, slots, experts, in, out, dtype, x_by_slot != 0, gradient != 0};
    if (!z.ok()) return 0;
    const ProductPlan p = product_plan(z, copies_matrices(w, ld_w, step_w, in, dtype), nullptr);
    return launches_fit(z, p) ? p.bytes : 0;
}

int iwp_expert_product(const void* x, int64_t ld_x, uint32_t x_by_slot, const void* w, int64_t ld_w, int64_t step_w, uint32_t tokens, uint32_t slots,
                       uint32_t experts, uint32_t in, uint32_t out, uint32_t dtype, const int32_t* chosen, void* y, int64_t ld_y, void* workspace,
                       size_t workspace_bytes, void* hip_stream) {
    const ProductSizes z{tokens, slots, experts, in, out, dtype, x_by_slot != 0, false};
    if (int rc = product_checks(z, x_by_slot, x, ld_x, w, ld_w, step_w, chosen)) return rc;
    if ((tokens && !y) || ld_y < out) return IWP_EINVAL;
    if (too_far(ld_x, dtype) || too_far(ld_w, dtype) || too_far(ld_y, dtype)) return IWP_ERANGE;
    const size_t e = size_of(dtype);
    if (!aligned(x, e) || !aligned(w, e) || !aligned(y, e) || !aligned(chosen, 4) || !aligned(workspace, 256)) return IWP_EALIGN;
    if (tokens == 0) return IWP_OK;
    const ProductPlan p = product_plan(z, copies_matrices(w, ld_w, step_w, in, dtype), workspace);
    if (!workspace || workspace_bytes < p.bytes) return IWP_EWORKSPACE;
    const hipStream_t s = static_cast<hipStream_t>(hip_stream);
    return with_kind(dtype, [&](auto kind) {
        typedef decltype(kind) K;
        constexpr int SIZE = K::E::SIZE;
        const RowsOut Y{static_cast<char*>(y), ld_y};
        if (few_rows(z)) {
            const bool by_slot = z.rows() <= experts;
            const uint32_t blocks = (out + FEW_ROWS - 1) / FEW_ROWS * (by_slot ? z.rows() : experts + 1);
            IWP_LAUNCH_BLOCK("k_expert_few", (k_expert_few<typename K::FEW_E, K::OUT>), blocks, 256, s,
                             (Matrices{static_cast<const char*>(w), step_w, (uint32_t)ld_w, out, in}),
                             (Packed{static_cast<const char*>(x), (uint32_t)ld_x, in, z.by_slot ? 1 : slots}), chosen, z.rows(), experts, by_slot, Y);
            return (int)IWP_OK;
        }
        // rows where they lie, else copied side by side, or gathered where 32 bits do not reach all of them
        const uint32_t per_row = z.by_slot ? 1 : slots, rows = z.rows() / per_row;
        Matrices W;
        Packed X{static_cast<const char*>(x), (uint32_t)ld_x, in, per_row};
        MatrixCopy copy{static_cast<const char*>(x), ld_x, 0, rows, in, Units{1, 0}, p.x};
        const bool lies = in_place(x, ld_x, in, rows, dtype), copied = !lies && in_place(p.x, p.ld_x, p.ld_x, rows, dtype);
        if (copied) copy.of = Units{p.ld_x * SIZE / 16, rows};
        if (!lies) X = Packed{p.x, p.ld_x, in, copied ? per_row : 0};
        int rc = arrange<SIZE>(z, p, chosen, w, ld_w, step_w, true, &W, copy, s);
        if (!rc && !X.slots) rc = gather<SIZE>(z, p, gather_of(z, x, ld_x, in, per_row, p.x, p.ld_x), RowsGather{}, s);
        if (rc) return rc;
        return with_lane<K>(readable(w, ld_w, step_w, in, dtype), [&](auto lane) {
            return with_tile_of<K>(p.tile, [&](auto tile) {
                typedef decltype(tile) T;
                auto kernel = X.slots ? k_expert_rows<typename K::E, T::BP, T::BQ, T::WP, T::WQ, K::OUT, false, decltype(lane)::value>
                                      : k_expert_rows<typename K::E, T::BP, T::BQ, T::WP, T::WQ, K::OUT, true, decltype(lane)::value>;
                const uint32_t more = T::BQ == Big::BQ ? MOST_HALVES : 0;
                IWP_LAUNCH_BLOCK("k_expert_rows", kernel, (out + T::BP - 1) / T::BP * p.max_tiles + more, T::THREADS, s, W, X, p.R, experts, Y);
                return (int)IWP_OK;
            });
        });
    });
}

int iwp_expert_product_gradient(const void* x, int64_t ld_x, uint32_t x_by_slot, const void* w, int64_t ld_w, int64_t step_w, uint32_t tokens,
                                uint32_t slots, uint32_t experts, uint32_t in, uint32_t out, uint32_t dtype, const int32_t* chosen, const void* dy,
                                int64_t ld_dy, void* dx, int64_t ld_dx, void* dw, int64_t ld_dw, int64_t step_dw, uint32_t dw_dtype, void* workspace,
                                size_t workspace_bytes, void* hip_stream) {
    const ProductSizes z{tokens, slots, experts, in, out, dtype, x_by_slot != 0, true};
    if (int rc = product_checks(z, x_by_slot, x, ld_x, w, ld_w, step_w, chosen)) return rc;
    if (dw && dw_dtype != dtype && dw_dtype != IWP_F32) return IWP_EINVAL;
    if ((tokens && !dy) || ld_dy < out || (dx && ld_dx < in)) return IWP_EINVAL;
    if (dw && (ld_dw < in || (experts > 1 && step_dw < (int64_t)(out - 1) * ld_dw + in))) return IWP_EINVAL;
    if (too_far(ld_x, dtype) || too_far(ld_w, dtype) || too_far(ld_dy, dtype) || (dx && too_far(ld_dx, dtype)) || (dw && too_far(ld_dw, dw_dtype)))
        return IWP_ERANGE;
    const size_t e = size_of(dtype);
    if (!aligned(x, e) || !aligned(w, e) || !aligned(dy, e) || !aligned(dx, e) || !aligned(dw, size_of(dw ? dw_dtype : dtype)) || !aligned(chosen, 4) ||
        !aligned(workspace, 256))
        return IWP_EALIGN;
    if ((tokens == 0 || !dx) && !dw) return IWP_OK;
    const ProductPlan p = product_plan(z, copies_matrices(w, ld_w, step_w, in, dtype), workspace);
    if (!workspace || workspace_bytes < p.bytes) return IWP_EWORKSPACE;
    const hipStream_t s = static_cast<hipStream_t>(hip_stream);
    return with_kind(dtype, [&](auto kind) {
        typedef decltype(kind) K;
        constexpr int SIZE = K::E::SIZE;
        const Packed X{p.x, p.ld_x, in, 0}, D{p.d, p.ld_d, out, 0};
        Matrices W;
        int rc = arrange<SIZE>(z, p, chosen, w, ld_w, step_w, dx && tokens, &W, MatrixCopy{}, s);
        if (!rc)
            rc = gather<SIZE>(z, p, gather_of(z, dy, ld_dy, out, 1, p.d, p.ld_d), dw ? gather_of(z, x, ld_x, in, z.by_slot ? 1 : slots, p.x, p.ld_x) : RowsGather{}, s);
        if (rc) return rc;
        // out_x, out_w: constants with the types of what the kernel writes
        auto products = [&](auto out_x, auto out_w) {
            return with_lane<K>(readable(w, ld_w, step_w, in, dtype), [&](auto lane) {
                return with_tile_of<K>(p.tile, [&](auto tile) {
                    typedef decltype(tile) T;
                    auto kernel = k_expert_gradients<typename K::E, T::BP, T::BQ, T::WP, T::WQ, decltype(out_x)::value, decltype(out_w)::value, decltype(lane)::value>;
                    const RowsOut rows = p.sums ? RowsOut{reinterpret_cast<char*>(p.sums), (int64_t)p.ld_x} : RowsOut{static_cast<char*>(dx), ld_dx};
                    const uint32_t tiles = dx ? (in + T::BP - 1) / T::BP * p.max_tiles : 0, matrices = dw ? (uint32_t)(experts * tiles_of<T>(in, out)) : 0;
                    IWP_LAUNCH_BLOCK("k_expert_gradients", kernel, ((tiles + 7) / 8 + 1 + (matrices + 7) / 8) * 8, T::THREADS, s, W, X, D, p.R, experts, rows,
                                     dx && tokens, dx && tokens && !p.sums, (MatricesOut{static_cast<char*>(dw), ld_dw, step_dw}), matrices);
                    return (int)IWP_OK;
                });
            });
        };
        constexpr std::integral_constant<int, K::OUT> own{};
        constexpr std::integral_constant<int, OUT_F32> wide{};
        const bool wide_w = dw && dw_dtype == IWP_F32;
        if (p.sums) rc = wide_w ? products(wide, wide) : products(wide, own);
        else rc = wide_w ? products(own, wide) : products(own, own);
        if (rc || !dx || !p.sums) return rc;
        const Spread sp = spread((in + 3) / 4);
        return in_launches(tokens, sp.rows(), sp.across, 256, [&](uint32_t first, uint32_t blocks) {
            IWP_LAUNCH_BLOCK("k_expert_sum", k_expert_sum<K::OUT>, blocks, 256, s, p.sums, p.ld_x, chosen, tokens, slots, experts, in, first, sp, dx, ld_dx);
            return (int)IWP_OK;
        });
    });
}

}  // extern "C"
