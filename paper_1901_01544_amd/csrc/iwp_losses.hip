// Host side of the C ABI declared in include/iwp_losses.h: argument checks, workspace carving and the launch sequences of the head's
// losses and of the expert balance.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "iwp_balance.hpp"
#include "iwp_head.hpp"
#include "iwp_host.hpp"

using namespace iwp;

namespace {

constexpr uint32_t TILE_ROWS = 256, TILE_VOCAB = 256;
constexpr uint32_t GROUP = 128;                    // vocabulary entries that share a largest logit and a sum
constexpr uint32_t CUS = 256;

struct Carver {            // hands out 256-byte aligned parts; at == nullptr: only adds up
    char* at;
    size_t used = 0;
    template <class T>
    void take(T*& p, size_t n) {
        p = at ? reinterpret_cast<T*>(at + used) : nullptr;
        used += (n * sizeof(T) + 255) & ~size_t(255);
    }
};

template <class T>
T round_up(T x, T to) { return (x + to - 1) / to * to; }

inline bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
inline size_t size_of(uint32_t dtype) { return dtype == IWP_F32 ? 4 : 2; }

// What a call of the head works with, from the sizes alone and whether the weight can be read where it lies.
struct HeadPlan {
    uint32_t tokens, dim, vocab, dtype, top, piece, pieces;
    uint32_t rows;         // tokens, rounded up to a tile
    uint32_t dim_padded;   // dim, rounded up to the LDS tile
    uint32_t ld_logits, ld_sums, splits, per_split, groups;
    bool f32, wide, copy_w;

    HeadScalars* scalars;
    HeadRows R;
    HeadStats St;
    Teacher T;
    uint16_t *h_hi, *h_lo, *w_hi, *w_lo, *g_hi, *g_lo;
    float* sums;
    size_t bytes;
};

bool readable(const void* w, int64_t ld_w, uint32_t dim, uint32_t dtype) {
    return dtype != IWP_F32 && aligned(w, 16) && ld_w % 8 == 0 && dim % 8 == 0;
}

constexpr uint32_t MAX_SPLITS = 32;

HeadPlan head_plan(uint32_t tokens, uint32_t dim, uint32_t vocab, uint32_t dtype, bool copy_w, uint32_t top, uint32_t piece,
                   void* workspace) {
    HeadPlan p{};
    p.tokens = tokens; p.dim = dim; p.vocab = vocab; p.dtype = dtype; p.top = top; p.copy_w = copy_w;
    p.f32 = dtype == IWP_F32;
    p.wide = dtype != IWP_BF16;
    p.piece = piece == 0 || piece >= vocab ? vocab : std::min(vocab, round_up(piece, TILE_VOCAB));
    p.pieces = (vocab + p.piece - 1) / p.piece;
    p.rows = round_up(std::max(tokens, 1u), TILE_ROWS);
    p.dim_padded = round_up(dim, BK);
    p.ld_logits = round_up(p.piece, TILE_VOCAB);
    p.ld_sums = copy_w ? p.dim_padded : dim;
    p.groups = (uint32_t)(((uint64_t)p.pieces * p.ld_logits + GROUP - 1) / GROUP);
    // dH has few tiles and a long sum: its vocabulary is split until every compute unit has a tile, at least 8 LDS tiles each
    const uint32_t tiles = (p.rows / TILE_ROWS) * ((dim + 255) / 256), steps = (p.piece + BK - 1) / BK;
    p.splits = std::max(1u, std::min({(CUS + tiles - 1) / tiles, steps / 8, MAX_SPLITS}));
    p.per_split = round_up((steps + p.splits - 1) / p.splits, 1u) * BK;

    Carver c{static_cast<char*>(workspace)};
    c.take(p.scalars, 1);
    c.take(p.R.token, p.rows);
    c.take(p.R.row, p.rows);
    c.take(p.R.label, p.rows);
    c.take(p.R.hard, p.rows);
    c.take(p.R.soft, p.rows);
    c.take(p.R.z_label, p.rows);
    c.take(p.R.lse, p.rows);
    c.take(p.R.lse_t, p.rows);
    p.St.ld = p.rows;
    c.take(p.St.m, (size_t)p.groups * p.rows);
    c.take(p.St.sum, (size_t)p.groups * p.rows);
    if (top) {
        c.take(p.St.sum_t, (size_t)p.groups * p.rows);
        c.take(p.T.index, (size_t)tokens * top);
        c.take(p.T.q, (size_t)tokens * top);
        c.take(p.T.z, (size_t)tokens * top);
        c.take(p.T.entropy, tokens);
        c.take(p.T.any, tokens);
        p.T.top = top;
    }
    c.take(p.h_hi, (size_t)p.rows * p.dim_padded);
    if (p.f32) c.take(p.h_lo, (size_t)p.rows * p.dim_padded);
    if (copy_w) c.take(p.w_hi, (size_t)vocab * p.dim_padded);
    if (p.f32) c.take(p.w_lo, (size_t)vocab * p.dim_padded);
    c.take(p.g_hi, (size_t)p.rows * p.ld_logits);
    if (p.wide) c.take(p.g_lo, (size_t)p.rows * p.ld_logits);
    c.take(p.sums, (size_t)p.splits * p.rows * p.ld_sums);
    p.bytes = c.used;
    return p;
}

bool sizes_ok(uint32_t tokens, uint32_t dim, uint32_t vocab, uint32_t dtype, uint32_t top) {
    return tokens <= IWP_MAX_TOKENS && dim >= 1 && dim <= IWP_MAX_DIM && vocab >= 1 && vocab <= IWP_MAX_VOCAB && dtype <= IWP_F16 &&
           top <= IWP_MAX_TOP;
}

struct HeadCall {
    const void *h, *w;
    int64_t ld_h, ld_w;
    const int32_t *top_index, *target;
    const float *top_logit, *weight;
    float temperature, soft, hard, scale;
    float* loss;
    void *dh, *dw;
    int64_t ld_dh, ld_dw;
    uint32_t dw_dtype;
    hipStream_t s;
};

struct KindF32 { typedef F16 E; typedef F32Element V; static constexpr bool F32 = true, WIDE = true; static constexpr int OUT = OUT_F32; };
struct KindBf16 { typedef Bf16 E; typedef Bf16 V; static constexpr bool F32 = false, WIDE = false; static constexpr int OUT = OUT_BF16; };
struct KindF16 { typedef F16 E; typedef F16 V; static constexpr bool F32 = false, WIDE = true; static constexpr int OUT = OUT_F16; };

struct Big { static constexpr int BP = 256, BQ = 256, WP = 2, WQ = 4, THREADS = 512; };

template <class K, class T, int MODE, bool SOFT>
int launch_logits(const HeadPlan& p, const HeadCall& c, const Operand& W, const Operand& H, const HeadPiece& G) {
    static_assert(T::BP / T::WP == GROUP, "a wavefront has a group");
    const uint32_t tiles = (G.n + T::BP - 1) / T::BP * (p.rows / T::BQ);
    auto kernel = k_head_logits<typename K::E, T::BP, T::BQ, T::WP, T::WQ, MODE, K::F32, K::WIDE, SOFT>;
    IWP_LAUNCH_BLOCK("k_head_logits", kernel, tiles, T::THREADS, c.s, W, H, p.dim_padded, G, p.R, p.St, c.temperature, p.scalars);
    return IWP_OK;
}

template <class K, class T, int OUT>
int launch_dw(const HeadPlan& p, const HeadCall& c, const Operand& H, const Operand& G, uint32_t first) {
    const uint32_t tiles = (p.dim + T::BP - 1) / T::BP * ((G.extent + T::BQ - 1) / T::BQ);
    auto kernel = k_head_dw<typename K::E, T::BP, T::BQ, T::WP, T::WQ, OUT, K::F32>;
    IWP_LAUNCH_BLOCK("k_head_dw", kernel, tiles, T::THREADS, c.s, H, G, c.scale, c.dw, c.ld_dw,
                     aligned(c.dw, 4) && c.ld_dw % 2 == 0, first, p.dim, p.scalars);
    return IWP_OK;
}

template <class K, bool SOFT>
int head(const HeadPlan& p, const HeadCall& c) {
    typedef Big T;
    const uint32_t tokens = std::max(p.tokens, 1u);        // grids: without tokens, the weight's gradient is still written
    Teacher teacher = p.T;
    teacher.t = c.temperature;
    if (SOFT) IWP_LAUNCH_BLOCK("k_head_teacher", k_head_teacher, (tokens + 3) / 4, 256, c.s, c.top_index, c.top_logit, p.tokens,
                               p.vocab, teacher);
    IWP_LAUNCH_BLOCK("k_head_rows", k_head_rows, 1, 1024, c.s, c.target, c.weight, SOFT ? p.T.any : nullptr, p.tokens, p.vocab, c.hard,
                     c.soft, c.temperature, p.R, c.loss, p.scalars);
    const uint32_t* count = &p.scalars->count;
    if (K::F32) {
        IWP_LAUNCH_BLOCK("k_head_max", k_head_max, std::min(tokens, 1024u), 256, c.s, static_cast<const float*>(c.h), c.ld_h, 0u, p.dim,
                         p.R.token, count, &p.scalars->h_max);
        IWP_LAUNCH_BLOCK("k_head_max", k_head_max, std::min(p.vocab, 2048u), 256, c.s, static_cast<const float*>(c.w), c.ld_w, p.vocab, p.dim,
                         (const uint32_t*)nullptr, (const uint32_t*)nullptr, &p.scalars->w_max);
    }
    IWP_LAUNCH_BLOCK("k_head_pack", k_head_pack<K::F32>, std::min(p.rows, 4096u), 256, c.s, c.h, c.ld_h, 0u, p.dim, p.R.token, count,
                     &p.scalars->h_max, p.h_hi, p.h_lo, p.dim_padded);
    if (p.copy_w)
        IWP_LAUNCH_BLOCK("k_head_pack", k_head_pack<K::F32>, std::min(p.vocab, 8192u), 256, c.s, c.w, c.ld_w, p.vocab, p.dim,
                         (const uint32_t*)nullptr, (const uint32_t*)nullptr, &p.scalars->w_max, p.w_hi, p.w_lo, p.dim_padded);
    const uint16_t* w_hi = p.copy_w ? p.w_hi : static_cast<const uint16_t*>(c.w);
    const size_t ld_w = p.copy_w ? p.dim_padded : (size_t)c.ld_w;
    const uint32_t dim_w = p.copy_w ? p.dim_padded : p.dim;
    const Operand H{p.h_hi, p.h_lo, p.dim_padded, p.rows, p.dim_padded};
    auto piece = [&](uint32_t i) {
        const uint32_t first = i * p.piece;
        return HeadPiece{first, std::min(p.piece, p.vocab - first), p.ld_logits, p.g_hi, p.g_lo};
    };
    auto weight = [&](const HeadPiece& G) {
        return Operand{w_hi + G.first * ld_w, p.w_lo ? p.w_lo + G.first * ld_w : nullptr, (uint32_t)ld_w, G.n, dim_w};
    };
    const bool gradients = c.dh || c.dw;
    int rc;
    for (uint32_t i = 0; i < p.pieces; ++i) {
        const HeadPiece G = piece(i);
        rc = i + 1 == p.pieces && gradients ? launch_logits<K, T, STATISTICS_KEPT, SOFT>(p, c, weight(G), H, G)
                                            : launch_logits<K, T, STATISTICS, SOFT>(p, c, weight(G), H, G);
        if (rc) return rc;
    }
    if (SOFT)
        IWP_LAUNCH_BLOCK("k_head_picked", k_head_picked<typename K::V>, (uint32_t)std::min<uint64_t>(((uint64_t)tokens * p.top + 3) / 4, 65536u),
                         256, c.s, c.h, c.ld_h, c.w, c.ld_w, p.dim, p.R, teacher, p.scalars);
    const uint32_t groups = (p.vocab + GROUP - 1) / GROUP;
    IWP_LAUNCH_BLOCK("k_head_join", k_head_join<SOFT>, (tokens + 31) / 32, 256, c.s, p.St, groups, p.R, teacher, c.loss, p.scalars);
    if (!gradients) return IWP_OK;
    for (uint32_t i = p.pieces; i-- > 0;) {
        const HeadPiece G = piece(i);
        const bool kept = i + 1 == p.pieces;
        if (kept) {
            auto kernel = k_head_dz<typename K::E, K::F32, K::WIDE, SOFT>;
            IWP_LAUNCH_BLOCK("k_head_dz", kernel, (p.ld_logits + 2047) / 2048 * p.rows, 256, c.s, G, GROUP, p.St, p.R,
                             c.temperature, p.scalars);
        } else if ((rc = launch_logits<K, T, GRADIENT, SOFT>(p, c, weight(G), H, G))) {
            return rc;
        }
        auto targets = k_head_targets<typename K::E, K::F32, SOFT>;
        IWP_LAUNCH_BLOCK("k_head_targets", targets, (uint32_t)std::min<uint64_t>(((uint64_t)tokens * (p.top + 1) + 255) / 256, 65536u), 256,
                         c.s, G, p.R, teacher, c.temperature, p.scalars);
        const uint16_t* g_lo = K::F32 ? p.g_lo : nullptr;
        if (c.dh) {
            Operand W = weight(G);
            W.extent = dim_w;
            W.summed = G.n;
            const Operand dz{p.g_hi, g_lo, p.ld_logits, p.rows, p.ld_logits};
            const uint32_t tiles = (dim_w + T::BP - 1) / T::BP * (p.rows / T::BQ);
            auto kernel = k_head_dh<typename K::E, T::BP, T::BQ, T::WP, T::WQ>;
            IWP_LAUNCH_BLOCK("k_head_dh", kernel, tiles * p.splits, T::THREADS, c.s, W, dz, p.splits, p.per_split, p.sums, p.ld_sums, !kept,
                             p.scalars);
        }
        if (c.dw) {
            const Operand Hc{p.h_hi, p.h_lo, p.dim_padded, p.dim_padded, 0u}, dz{p.g_hi, g_lo, p.ld_logits, G.n, 0u};
            rc = c.dw_dtype == IWP_F32 ? launch_dw<K, T, OUT_F32>(p, c, Hc, dz, G.first) : launch_dw<K, T, K::OUT>(p, c, Hc, dz, G.first);
            if (rc) return rc;
        }
    }
    if (c.dh && p.tokens)
        IWP_LAUNCH_BLOCK("k_head_dh_out", (k_head_dh_out<K::OUT, K::F32>), tokens, 256, c.s, p.sums, p.splits, p.rows, p.ld_sums, p.R, p.dim,
                         c.scale, c.dh, c.ld_dh, p.scalars);
    return IWP_OK;
}

int head_call(const HeadCall& c, uint32_t tokens, uint32_t dim, uint32_t vocab, uint32_t dtype, uint32_t top, uint32_t piece, void* workspace,
              size_t workspace_bytes) {
    if (!sizes_ok(tokens, dim, vocab, dtype, top)) return IWP_EINVAL;
    if (c.dw && c.dw_dtype != dtype && c.dw_dtype != IWP_F32) return IWP_EINVAL;
    if (!std::isfinite(c.scale) || !std::isfinite(c.hard) || !std::isfinite(c.soft) || !(c.temperature > 0.0f) || !std::isfinite(c.temperature))
        return IWP_EINVAL;
    if (tokens && (!c.h || !c.loss)) return IWP_EINVAL;
    if (!c.w) return IWP_EINVAL;
    if (c.ld_h < dim || c.ld_w < dim || (c.dh && c.ld_dh < dim) || (c.dw && c.ld_dw < dim)) return IWP_EINVAL;
    if (c.ld_h >= 1 << 23 || c.ld_w >= 1 << 23 || (c.dh && c.ld_dh >= 1 << 23) || (c.dw && c.ld_dw >= 1 << 23)) return IWP_ERANGE;
    const size_t e = size_of(dtype);
    if (!aligned(c.h, e) || !aligned(c.w, e) || !aligned(c.dh, e) || !aligned(c.dw, size_of(c.dw ? c.dw_dtype : dtype)) || !aligned(c.loss, 4) ||
        !aligned(c.target, 4) || !aligned(c.weight, 4) || !aligned(c.top_index, 4) || !aligned(c.top_logit, 4) || !aligned(workspace, 256))
        return IWP_EALIGN;
    if (tokens == 0 && !c.dw) return IWP_OK;
    const HeadPlan p = head_plan(tokens, dim, vocab, dtype, !readable(c.w, c.ld_w, dim, dtype), top, piece, workspace);
    if (!workspace || workspace_bytes < p.bytes) return IWP_EWORKSPACE;
    if (top) {
        if (dtype == IWP_F32) return head<KindF32, true>(p, c);
        return dtype == IWP_BF16 ? head<KindBf16, true>(p, c) : head<KindF16, true>(p, c);
    }
    if (dtype == IWP_F32) return head<KindF32, false>(p, c);
    return dtype == IWP_BF16 ? head<KindBf16, false>(p, c) : head<KindF16, false>(p, c);
}

constexpr uint32_t BALANCE_GROUPS = 512;

uint32_t balance_groups(uint32_t tokens) { return std::max(1u, std::min(BALANCE_GROUPS, (tokens + 3) / 4)); }

size_t balance_carve(BalanceSums* B, uint32_t groups, uint32_t experts, void* workspace) {
    Carver c{static_cast<char*>(workspace)};
    c.take(B->p, (size_t)groups * experts);
    c.take(B->slots, (size_t)groups * experts);
    c.take(B->square, groups);
    c.take(B->tokens, groups);
    c.take(B->p_all, experts);
    c.take(B->square_all, 1);
    c.take(B->tokens_all, 1);
    return c.used;
}

template <int IN, int NV>
int balance_run(const void* x, int64_t ld_x, uint32_t tokens, uint32_t experts, const int32_t* chosen, uint32_t slots, const uint8_t* keep,
                float balance, float z, float* loss, int32_t* counts, void* dx, int64_t ld_dx, const BalanceSums& B, uint32_t groups,
                hipStream_t s) {
    auto rows = k_balance_rows<IN, NV>;
    auto grad = k_balance_grad<IN, NV>;
    IWP_LAUNCH_BLOCK("k_balance_rows", rows, groups, 256, s, x, ld_x, tokens, experts, chosen, slots, keep, B);
    IWP_LAUNCH_BLOCK("k_balance_join", k_balance_join, experts / 4 + 1, 256, s, B, groups, experts, counts);
    IWP_LAUNCH_BLOCK("k_balance_grad", grad, dx ? std::max(1u, std::min((tokens + 3) / 4, 2048u)) : 1u, 256, s, x, ld_x, tokens, experts, slots,
                     keep, balance, z, B, counts, loss, dx, ld_dx);
    return IWP_OK;
}

template <int IN, class... A>
int balance_typed(uint32_t experts, A... a) {
    if (experts <= 64) return balance_run<IN, 1>(a...);
    if (experts <= 128) return balance_run<IN, 2>(a...);
    if (experts <= 256) return balance_run<IN, 4>(a...);
    if (experts <= 512) return balance_run<IN, 8>(a...);
    return balance_run<IN, 16>(a...);
}

}  // namespace

extern "C" {

size_t iwp_head_workspace_bytes(uint32_t tokens, uint32_t dim, uint32_t vocab, uint32_t dtype, const void* w, int64_t ld_w, uint32_t top,
                                uint32_t piece) {
    if (!sizes_ok(tokens, dim, vocab, dtype, top)) return 0;
    return head_plan(tokens, dim, vocab, dtype, !readable(w, ld_w, dim, dtype), top, piece, nullptr).bytes;
}

int iwp_head_cross_entropy(const void* h, int64_t ld_h, const void* w, int64_t ld_w, uint32_t tokens, uint32_t dim, uint32_t vocab,
                           uint32_t dtype, const int32_t* target, const float* weight, float scale, uint32_t piece, float* loss, void* dh,
                           int64_t ld_dh, void* dw, int64_t ld_dw, uint32_t dw_dtype, void* workspace, size_t workspace_bytes,
                           void* hip_stream) {
    if (tokens && !target) return IWP_EINVAL;
    const HeadCall c{h, w, ld_h, ld_w, nullptr, target, nullptr, weight, 1.0f, 0.0f, 1.0f, scale, loss, dh, dw, ld_dh, ld_dw, dw_dtype,
                     static_cast<hipStream_t>(hip_stream)};
    return head_call(c, tokens, dim, vocab, dtype, 0, piece, workspace, workspace_bytes);
}

int iwp_head_distill(const void* h, int64_t ld_h, const void* w, int64_t ld_w, uint32_t tokens, uint32_t dim, uint32_t vocab, uint32_t dtype,
                     const int32_t* top_index, const float* top_logit, uint32_t top, float temperature, float soft, const int32_t* target,
                     float hard, const float* weight, float scale, uint32_t piece, float* loss, void* dh, int64_t ld_dh, void* dw,
                     int64_t ld_dw, uint32_t dw_dtype, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (top == 0 || (tokens && (!top_index || !top_logit))) return IWP_EINVAL;
    const HeadCall c{h, w, ld_h, ld_w, top_index, target, top_logit, weight, temperature, soft, hard, scale, loss, dh, dw, ld_dh, ld_dw,
                     dw_dtype, static_cast<hipStream_t>(hip_stream)};
    return head_call(c, tokens, dim, vocab, dtype, top, piece, workspace, workspace_bytes);
}

size_t iwp_balance_workspace_bytes(uint32_t tokens, uint32_t experts) {
    if (tokens > IWP_MAX_TOKENS || experts < 1 || experts > IWP_MAX_EXPERTS) return 0;
    BalanceSums B{};
    return balance_carve(&B, balance_groups(tokens), experts, nullptr);
}

int iwp_balance(const void* x, int64_t ld_x, uint32_t tokens, uint32_t experts, uint32_t dtype, const int32_t* chosen, uint32_t slots,
                const uint8_t* keep, float balance, float z, float* loss, int32_t* counts, void* dx, int64_t ld_dx, void* workspace,
                size_t workspace_bytes, void* hip_stream) {
    if (tokens > IWP_MAX_TOKENS || experts < 1 || experts > IWP_MAX_EXPERTS || dtype > IWP_F16 || slots < 1 || slots > experts) return IWP_EINVAL;
    if (!std::isfinite(balance) || !std::isfinite(z) || !loss || !counts || (tokens && (!x || !chosen))) return IWP_EINVAL;
    if (ld_x < experts || (dx && ld_dx < experts)) return IWP_EINVAL;
    const size_t e = size_of(dtype);
    if (!aligned(x, e) || !aligned(dx, e) || !aligned(chosen, 4) || !aligned(loss, 4) || !aligned(counts, 4) || !aligned(workspace, 256))
        return IWP_EALIGN;
    BalanceSums B{};
    const uint32_t groups = balance_groups(tokens);
    if (!workspace || workspace_bytes < balance_carve(&B, groups, experts, workspace)) return IWP_EWORKSPACE;
    const hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (dtype == IWP_F32)
        return balance_typed<OUT_F32>(experts, x, ld_x, tokens, experts, chosen, slots, keep, balance, z, loss, counts, dx, ld_dx, B, groups, s);
    if (dtype == IWP_BF16)
        return balance_typed<OUT_BF16>(experts, x, ld_x, tokens, experts, chosen, slots, keep, balance, z, loss, counts, dx, ld_dx, B, groups, s);
    return balance_typed<OUT_F16>(experts, x, ld_x, tokens, experts, chosen, slots, keep, balance, z, loss, counts, dx, ld_dx, B, groups, s);
}

}  // extern "C"
