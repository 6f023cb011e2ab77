// Host side of the C ABI declared in include/iwp_losses.h: argument checks, workspace carving and the launch sequences of the head's
// losses and of the expert balance.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "iwp_balance.hpp"
#include "iwp_head.hpp"
#include "iwp_host.hpp"
#include "iwp_launch_rows.hpp"

using namespace iwp;

namespace {

constexpr uint32_t TILE_VOCAB = 256;                 // pieces of the vocabulary start and end at multiples of the largest tile
constexpr uint32_t CUS = 256;

// Tiles of the products.  GROUP: vocabulary entries of a wavefront, which share a largest logit and a sum; RESIDENT: workgroups that a
// compute unit holds at a time.
struct Big { static constexpr int BP = 256, BQ = 256, WP = 2, WQ = 4, THREADS = 512, GROUP = BP / WP, RESIDENT = 1; };
struct Mid { static constexpr int BP = 128, BQ = 128, WP = 2, WQ = 2, THREADS = 256, GROUP = BP / WP; };
struct Few { static constexpr int BP = 64, BQ = 64, WP = 2, WQ = 2, THREADS = 256, GROUP = BP / WP, RESIDENT = 4; };
enum TileKind { BIG, MID, FEW };

template <class T>
uint32_t tiles_of(uint32_t np, uint32_t nq) { return (np + T::BP - 1) / T::BP * ((nq + T::BQ - 1) / T::BQ); }

// The largest tile of which there are enough for most of the 256 compute units.  us with the large tile and with the one taken: logits of
// 5 tokens x 768 x 8192 (32 large tiles, 128 small) 24.6 and 11.7, its dH 14.0 and 7.8; binary32 logits of 37 x 512 x 1000 (4, 16)
// 34.9 and 16.7, its dH 30.5 and 16.1, its dW (8, 128) 11.0 and 4.7; dW of 800 x 640 x 10007 (120 large, 395 middling) 60.2 and
// 40.5.  At the limit, logits and dW of 1024 tokens x 1024 in bf16, large tiles and middling ones (small):
//   64 large tiles   33 and 29   21 and 20 (24 and 24)        160   33 and 29   36 and 34
//   128              33 and 29   26 and 24                    192   35 and 31   36 and 34      256   39 and 36   43 and 40
// in binary32 96 tiles 65, 50; 160 tiles 72, 87.  (Two middling tiles fit a compute unit: 128 large ones make 512, one round of the chip.)
constexpr uint32_t ENOUGH_TILES = 160;
TileKind tile_for(uint32_t np, uint32_t nq) {
    if (tiles_of<Big>(np, nq) >= ENOUGH_TILES) return BIG;
    return tiles_of<Mid>(np, nq) >= ENOUGH_TILES ? MID : FEW;
}

// f(tile) with the tile's type
template <class F>
int with_tile(TileKind kind, F f) {
    switch (kind) {
        case BIG: return f(Big{});
        case MID: return f(Mid{});
        default: return f(Few{});
    }
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

template <class T>
T round_up(T x, T to) { return (x + to - 1) / to * to; }

inline bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
inline size_t size_of(uint32_t dtype) { return dtype == IWP_F32 ? 4 : 2; }

// What a call of the head works with, from the sizes alone and whether the weight can be read where it lies.
struct HeadPlan {
    uint32_t tokens, dim, vocab, dtype, top, piece, pieces;
    uint32_t rows;         // tokens, rounded up to a tile
    uint32_t dim_padded;   // dim, rounded up to the LDS tile
    uint32_t ld_logits, ld_sums, splits, per_split, group, groups;
    TileKind logits_tile, dh_tile;
    bool f32, wide, copy_w;

    HeadScalars* scalars;
    HeadRows R;
    HeadStats St;
    Teacher T;
    uint16_t *h_hi, *h_lo, *w_hi, *w_lo, *g_hi, *g_lo;
    uint16_t *hs_hi, *hs_lo;                             // h times powers of two for the tokens' coefficients
    float* sums;
    size_t bytes;
};

Spread spread(uint32_t units) {
    Spread s{0, 1};
    while (s.shift < 8 && (1u << s.shift) < units) ++s.shift;
    s.across = (units + (1u << s.shift) - 1) >> s.shift;
    return s;
}

bool readable(const void* w, int64_t ld_w, uint32_t dim, uint32_t dtype) {
    return dtype != IWP_F32 && aligned(w, 16) && ld_w % 8 == 0 && dim % 8 == 0;
}

// A split's sums are tokens x dim in binary32, written and read again.  dH and the joining of its sums, us, with 16, 32 and 64 splits at most: 64
// tokens x 1024 x 131072 107, 73, 92; 100 x 512 x 131072 156, 89, 59; 256 x 1024 x 131072 207, 134, 118; 64 x 512 x 32768 30, 24, 27.
constexpr uint32_t MAX_SPLITS = 32;

uint32_t held(uint32_t vocab, uint32_t piece) {         // entries of the vocabulary whose logits are held at a time
    return piece == 0 || piece >= vocab ? vocab : std::min(vocab, round_up(piece, TILE_VOCAB));
}

HeadPlan head_plan(uint32_t tokens, uint32_t dim, uint32_t vocab, uint32_t dtype, bool copy_w, uint32_t top, uint32_t piece,
                   void* workspace) {
    HeadPlan p{};
    p.tokens = tokens; p.dim = dim; p.vocab = vocab; p.dtype = dtype; p.top = top; p.copy_w = copy_w;
    p.T.t = 1.0f;
    p.f32 = dtype == IWP_F32;
    p.wide = dtype != IWP_BF16;
    p.piece = held(vocab, piece);
    p.pieces = (vocab + p.piece - 1) / p.piece;
    p.rows = round_up(std::max(tokens, 1u), tokens <= Few::BQ ? (uint32_t)Few::BQ : (uint32_t)Big::BQ);
    p.dim_padded = round_up(dim, BK);
    p.ld_logits = round_up(p.piece, TILE_VOCAB);
    p.ld_sums = copy_w ? p.dim_padded : dim;
    p.logits_tile = p.rows < Big::BQ ? FEW : tile_for(p.piece, p.tokens);   // a tile's rows are all written
    p.group = p.logits_tile == BIG ? Big::GROUP : p.logits_tile == MID ? Mid::GROUP : Few::GROUP;
    p.groups = (uint32_t)(((uint64_t)p.pieces * p.ld_logits + p.group - 1) / p.group);
    // dH has few tiles and a long sum: its vocabulary is split until the compute units are full, at least 8 LDS tiles each.  Up to 64 tokens
    // small tiles, above that large ones: 64 x 512 x 32768 16 us, 100 x 512 x 32768 27 (small tiles 18), 200 x 768 x 32768 32 (35), 256 x 1024
    // x 131072 121 (181)
    const uint32_t steps = (p.piece + BK - 1) / BK;
    p.dh_tile = tokens <= Few::BQ ? FEW : BIG;
    const uint32_t tiles = std::max(1u, p.dh_tile == FEW ? tiles_of<Few>(dim, tokens) : tiles_of<Big>(dim, tokens));
    const uint32_t room = CUS * (p.dh_tile == FEW ? Few::RESIDENT : Big::RESIDENT);
    p.splits = std::max(1u, std::min({(room + tiles - 1) / tiles, steps / 8, MAX_SPLITS}));
    p.per_split = (steps + p.splits - 1) / p.splits * BK;

    Carver c{static_cast<char*>(workspace)};
    c.take(p.scalars, 1);
    c.take(p.R.token, p.rows);
    c.take(p.R.row, p.rows);
    c.take(p.R.label, p.rows);
    c.take(p.R.hard, p.rows);
    c.take(p.R.soft, p.rows);
    c.take(p.R.exponent, p.rows);
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
        p.T.width = TILE_VOCAB;
        while ((vocab + p.T.width - 1) / p.T.width > STRETCHES) p.T.width *= 2;
        p.T.stretches = (vocab + p.T.width - 1) / p.T.width;
        c.take(p.T.start, (size_t)((tokens + 63) / 64) * (p.T.stretches + 1));
        c.take(p.T.found, (size_t)((tokens + 63) / 64) * 64 * top);
    }
    c.take(p.h_hi, (size_t)p.rows * p.dim_padded);
    if (p.f32) c.take(p.h_lo, (size_t)p.rows * p.dim_padded);
    c.take(p.hs_hi, (size_t)p.rows * p.dim_padded);
    if (p.f32) c.take(p.hs_lo, (size_t)p.rows * p.dim_padded);
    if (copy_w) c.take(p.w_hi, (size_t)vocab * p.dim_padded);
    if (p.f32) c.take(p.w_lo, (size_t)vocab * p.dim_padded);
    c.take(p.g_hi, (size_t)p.rows * p.ld_logits);
    if (p.wide) c.take(p.g_lo, (size_t)p.rows * p.ld_logits);
    c.take(p.sums, (size_t)p.splits * p.rows * p.ld_sums);
    p.bytes = c.used;
    return p;
}

// Up to IWP_MAX_HELD logits at a time every product's launch stays below 2^31 threads: 512 for 256 x 256 logits or gradients (the smaller
// tiles are taken where tiles are few).
bool sizes_ok(uint32_t tokens, uint32_t dim, uint32_t vocab, uint32_t dtype, uint32_t top, uint32_t piece) {
    return tokens <= IWP_MAX_TOKENS && dim >= 1 && dim <= IWP_MAX_DIM && vocab >= 1 && vocab <= IWP_MAX_VOCAB && dtype <= IWP_F16 &&
           top <= IWP_MAX_TOP && (uint64_t)tokens * held(vocab, piece) <= IWP_MAX_HELD;
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

struct KindF32 { typedef F16 E; static constexpr bool F32 = true, WIDE = true; static constexpr int OUT = OUT_F32; };
struct KindBf16 { typedef Bf16 E; static constexpr bool F32 = false, WIDE = false; static constexpr int OUT = OUT_BF16; };
struct KindF16 { typedef F16 E; static constexpr bool F32 = false, WIDE = true; static constexpr int OUT = OUT_F16; };

template <class K, class T, int MODE, bool SOFT>
int launch_logits(const HeadPlan& p, const HeadCall& c, const Operand& W, Operand H, const HeadPiece& G) {
    H.extent = round_up(std::max(p.tokens, 1u), (uint32_t)T::BQ);
    auto kernel = k_head_logits<typename K::E, T::BP, T::BQ, T::WP, T::WQ, MODE, K::F32, K::WIDE, SOFT>;
    IWP_LAUNCH_BLOCK("k_head_logits", kernel, tiles_of<T>(G.n, H.extent), T::THREADS, c.s, W, H, p.dim_padded, G, p.R, p.St, p.T, p.scalars);
    return IWP_OK;
}

template <class K, int OUT>
int launch_dw(const HeadPlan& p, const HeadCall& c, const Operand& H, const Operand& G, uint32_t first) {
    return with_tile(tile_for(p.dim, G.extent), [&](auto tile) {
        typedef decltype(tile) T;
        auto kernel = k_head_dw<typename K::E, T::BP, T::BQ, T::WP, T::WQ, OUT, K::F32>;
        IWP_LAUNCH_BLOCK("k_head_dw", kernel, tiles_of<T>(p.dim, G.extent), T::THREADS, c.s, H, (Planes{p.hs_hi, p.hs_lo}), G, c.scale,
                         c.dw, c.ld_dw, first, p.dim, p.scalars);
        return (int)IWP_OK;
    });
}

template <class K, class T>
int launch_dh(const HeadPlan& p, const HeadCall& c, const Operand& W, Operand G, bool add) {
    G.extent = round_up(p.tokens, (uint32_t)T::BQ);
    auto kernel = k_head_dh<typename K::E, T::BP, T::BQ, T::WP, T::WQ>;
    IWP_LAUNCH_BLOCK("k_head_dh", kernel, tiles_of<T>(W.extent, G.extent) * p.splits, T::THREADS, c.s, W, G, p.splits, p.per_split, p.sums,
                     p.rows, p.ld_sums, add, p.scalars);
    return IWP_OK;
}

template <class K, bool SOFT>
int head(const HeadPlan& p, const HeadCall& c) {
    const uint32_t tokens = std::max(p.tokens, 1u);        // grids: without tokens, the weight's gradient is still written
    if (SOFT) IWP_LAUNCH_BLOCK("k_head_teacher", k_head_teacher, (tokens + 3) / 4, 256, c.s, c.top_index, c.top_logit, c.target, p.tokens,
                               p.vocab, p.T);
    IWP_LAUNCH_BLOCK("k_head_rows", k_head_rows, 1, 1024, c.s, c.target, c.weight, SOFT ? p.T.any : nullptr, p.tokens, p.vocab, c.hard,
                     c.soft, c.temperature, p.R, c.loss, p.scalars);
    if (SOFT) IWP_LAUNCH_BLOCK("k_head_sort", k_head_sort, (tokens + 63) / 64, 1024, c.s, p.R, p.T, p.scalars);
    const HeadMatrix h{c.h, c.ld_h, p.tokens, p.dim, p.R.token, &p.scalars->count}, w{c.w, c.ld_w, p.vocab, p.dim, nullptr, nullptr};
    // without weights and a teacher all coefficients are the same
    const bool scaled = c.dw && (SOFT || c.weight);
    constexpr bool IS_F16 = !K::F32 && std::is_same<typename K::E, F16>::value;
    if (K::F32 || (IS_F16 && scaled)) {
        auto blocks = [&](uint32_t rows, uint32_t most) { return std::max(1u, std::min((rows + 15) / 16 * ((p.dim + 1023) / 1024), most)); };
        const uint32_t hb = blocks(p.tokens, K::F32 ? 64 : 256), wb = K::F32 ? blocks(p.vocab, 256) : 0;
        IWP_LAUNCH_BLOCK("k_head_max", k_head_max<K::F32>, hb + wb, 1024, c.s, h, w, hb, p.scalars);
    }
    const Spread packed = spread(p.dim_padded / 8);
    auto pack = [&](auto kernel, const HeadMatrix& m, uint32_t rows, const uint32_t* max_bits, const Planes& to) {
        return in_launches(rows, packed.rows() * PACK_ROWS, packed.across, 256, [&](uint32_t first, uint32_t blocks) {
            IWP_LAUNCH_BLOCK("k_head_pack", kernel, blocks, 256, c.s, m, first, packed, max_bits, to, (Planes{p.hs_hi, p.hs_lo}), p.R.exponent,
                             p.dim_padded, p.scalars);
            return (int)IWP_OK;
        });
    };
    int rc = scaled ? pack(k_head_pack<typename K::E, K::F32, true>, h, p.rows, &p.scalars->h_max, Planes{p.h_hi, p.h_lo})
                    : pack(k_head_pack<typename K::E, K::F32, false>, h, p.rows, &p.scalars->h_max, Planes{p.h_hi, p.h_lo});
    if (!rc && p.copy_w) rc = pack(k_head_pack<typename K::E, K::F32, false>, w, p.vocab, &p.scalars->w_max, Planes{p.w_hi, p.w_lo});
    if (rc) return rc;
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
    for (uint32_t i = 0; i < p.pieces; ++i) {
        const HeadPiece G = piece(i);
        rc = with_tile(p.logits_tile, [&](auto tile) {
            typedef decltype(tile) T;
            return i + 1 == p.pieces && gradients ? launch_logits<K, T, STATISTICS_KEPT, SOFT>(p, c, weight(G), H, G)
                                                  : launch_logits<K, T, STATISTICS, SOFT>(p, c, weight(G), H, G);
        });
        if (rc) return rc;
    }
    const uint32_t groups = (p.vocab + p.group - 1) / p.group;
    IWP_LAUNCH_BLOCK("k_head_join", k_head_join<SOFT>, (tokens + 15) / 16, 512, c.s, p.St, groups, p.R, p.T, c.loss, p.scalars);
    if (!gradients) return IWP_OK;
    for (uint32_t i = p.pieces; i-- > 0;) {
        const HeadPiece G = piece(i);
        const bool kept = i + 1 == p.pieces;
        if (kept) {
            auto kernel = k_head_dz<typename K::E, K::F32, K::WIDE, SOFT>;
            rc = in_launches(p.rows, 1, (p.ld_logits + DZ_ACROSS - 1) / DZ_ACROSS, 256, [&](uint32_t first, uint32_t blocks) {
                IWP_LAUNCH_BLOCK("k_head_dz", kernel, blocks, 256, c.s, G, first, p.group, p.St, p.R, p.T, p.scalars);
                return (int)IWP_OK;
            });
            if (rc) return rc;
        } else {
            rc = p.rows < Big::BQ ? launch_logits<K, Few, GRADIENT, SOFT>(p, c, weight(G), H, G)
                                  : launch_logits<K, Big, GRADIENT, SOFT>(p, c, weight(G), H, G);
            if (rc) return rc;
        }
        if (SOFT || !kept) {
            auto targets = k_head_targets<typename K::E, K::F32, SOFT>;
            IWP_LAUNCH_BLOCK("k_head_targets", targets, (tokens + 3) / 4, 256, c.s, G, p.R, p.T, p.scalars);
        }
        const uint16_t* g_lo = K::F32 ? p.g_lo : nullptr;
        if (c.dh && p.tokens) {
            Operand W = weight(G);
            W.extent = dim_w;
            W.summed = G.n;
            const Operand dz{p.g_hi, g_lo, p.ld_logits, 0u, p.ld_logits};
            rc = p.dh_tile == FEW ? launch_dh<K, Few>(p, c, W, dz, !kept) : launch_dh<K, Big>(p, c, W, dz, !kept);
            if (rc) return rc;
        }
        if (c.dw) {
            const Operand Hc{p.h_hi, p.h_lo, p.dim_padded, p.dim_padded, 0u}, dz{p.g_hi, g_lo, p.ld_logits, G.n, 0u};
            rc = c.dw_dtype == IWP_F32 ? launch_dw<K, OUT_F32>(p, c, Hc, dz, G.first) : launch_dw<K, K::OUT>(p, c, Hc, dz, G.first);
            if (rc) return rc;
        }
    }
    const Spread out = spread((p.dim + 3) / 4);
    if (!c.dh) return IWP_OK;
    return in_launches(p.tokens, out.rows(), out.across, 256, [&](uint32_t first, uint32_t blocks) {
        IWP_LAUNCH_BLOCK("k_head_dh_out", (k_head_dh_out<K::OUT, K::F32>), blocks, 256, c.s, p.sums, p.splits, p.rows, p.ld_sums, p.R, first,
                         out, p.tokens, p.dim, c.scale, c.dh, c.ld_dh, p.scalars);
        return (int)IWP_OK;
    });
}

int head_call(const HeadCall& c, uint32_t tokens, uint32_t dim, uint32_t vocab, uint32_t dtype, uint32_t top, uint32_t piece, void* workspace,
              size_t workspace_bytes) {
    if (!sizes_ok(tokens, dim, vocab, dtype, top, piece)) return IWP_EINVAL;
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
    HeadPlan p = head_plan(tokens, dim, vocab, dtype, !readable(c.w, c.ld_w, dim, dtype), top, piece, workspace);
    p.T.t = c.temperature;
    if (!workspace || workspace_bytes < p.bytes) return IWP_EWORKSPACE;
    if (top) {
        if (dtype == IWP_F32) return head<KindF32, true>(p, c);
        return dtype == IWP_BF16 ? head<KindBf16, true>(p, c) : head<KindF16, true>(p, c);
    }
    if (dtype == IWP_F32) return head<KindF32, false>(p, c);
    return dtype == IWP_BF16 ? head<KindBf16, false>(p, c) : head<KindF16, false>(p, c);
}

constexpr uint32_t BALANCE_GROUPS = 512;
// One workgroup does it all where that is up to this many logits, 16 a lane of its 16 wavefronts, or all tokens at once.  us a call, and as
// three launches: 64 tokens x 8 experts in binary32 6.8 and 11.9; 16 logits a lane: 2048 x 8 11.3 and 11.8, 1024 x 9 12.8 and 11.8, 256 x 33
// in bf16 12.0 and 11.9; more, where tokens do not fill their lanes (a power of two, 16 bytes or more each): 1820 x 9 20 and 12, 16384 x 1
// 33 and 12, in bf16 50 and 12.  16 x 1024 at once 11.8 and 19.
constexpr uint64_t BALANCE_ONE = 16384;
constexpr uint32_t BALANCE_ONE_LANE = BALANCE_ONE / (BALANCE_ONE_WAVES * 64);

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

template <int IN, int CHUNKS>
int balance_run(const Router& r, const BalanceGradient& g, float* loss, int32_t* counts, const BalanceSums& B, uint32_t groups, hipStream_t s) {
    auto one = k_balance_one<IN, CHUNKS>;
    auto rows = k_balance_rows<IN, CHUNKS>;
    auto grad = k_balance_grad<IN, CHUNKS>;
    const uint32_t rounds = std::max(1u, BALANCE_ONE_LANE / TokenLanes<IN, CHUNKS>::N);
    if ((uint64_t)r.tokens * r.experts <= BALANCE_ONE && r.tokens <= rounds * BALANCE_ONE_WAVES * (64 / r.lanes)) {
        IWP_LAUNCH_BLOCK("k_balance_one", one, 1, BALANCE_ONE_WAVES * 64, s, r, g, counts, loss);
        return IWP_OK;
    }
    const uint32_t at_once = 4 * (64 / r.lanes), blocks = std::max(1u, (r.tokens + at_once - 1) / at_once);
    groups = std::min(groups, blocks);
    IWP_LAUNCH_BLOCK("k_balance_rows", rows, groups, 256, s, r, B);
    IWP_LAUNCH_BLOCK("k_balance_join", k_balance_join, r.experts / 4 + 1, 256, s, B, groups, r.experts, counts);
    IWP_LAUNCH_BLOCK("k_balance_grad", grad, g.dx ? std::min(blocks, 2048u) : 1u, 256, s, r, g, B, counts, loss);
    return IWP_OK;
}

// 16 bytes a lane up to 16 lanes a token, then two and four times as many bytes before more lanes: a token's sums take a step less
// for every halving of its lanes.
template <int IN>
int balance_typed(Router r, const BalanceGradient& g, float* loss, int32_t* counts, const BalanceSums& B, uint32_t groups, hipStream_t s) {
    const uint32_t units = (r.experts + TokenLanes<IN, 1>::WIDTH - 1) / TokenLanes<IN, 1>::WIDTH;
    const uint32_t chunks = units <= 16 ? 1 : units <= 32 ? 2 : 4;
    r.lanes = 1;
    while (r.lanes * chunks < units) r.lanes *= 2;
    if (chunks == 1) return balance_run<IN, 1>(r, g, loss, counts, B, groups, s);
    return chunks == 2 ? balance_run<IN, 2>(r, g, loss, counts, B, groups, s) : balance_run<IN, 4>(r, g, loss, counts, B, groups, s);
}

}  // namespace

extern "C" {

size_t iwp_head_workspace_bytes(uint32_t tokens, uint32_t dim, uint32_t vocab, uint32_t dtype, const void* w, int64_t ld_w, uint32_t top,
                                uint32_t piece) {
    if (!sizes_ok(tokens, dim, vocab, dtype, top, piece)) return 0;
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
    const Router r{x, ld_x, tokens, experts, 0, slots, chosen, keep};
    const BalanceGradient g{balance, z, dx, ld_dx};
    if (dtype == IWP_F32) return balance_typed<OUT_F32>(r, g, loss, counts, B, groups, s);
    return dtype == IWP_BF16 ? balance_typed<OUT_BF16>(r, g, loss, counts, B, groups, s) : balance_typed<OUT_F16>(r, g, loss, counts, B, groups, s);
}

}  // extern "C"
