// Kernels of the experts' products: which rows (slots of tokens) go to which expert, those rows side by side, and the products of every
// expert's rows with its matrix, one launch for all experts:
//   y_r = W_e x_r,  dx_r = W_e^T dy_r,  dW_e = sum over e's rows of dy_r x_r^T
//
// Bound by the matrix cores and, where matrices are many and rows few, by memory.  In bf16: 16384 rows, 8 x 2048 x 4096, 275 GFLOP in 265 to 277 us, the
// matrix cores busy 61 % of the cycles; both gradients of 32768 rows, 64 x 2048 x 1024, 275 GFLOP in 460 us, busy 36 %, 308 without their 805 MB of stores.
// Nothing hides the stores of either.  Binary32: 8192 rows, 8 x 1024 x 1024, 151 us, 114 TFLOP/s of 153.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/iwp_experts.h"
#include "iwp_halves.hpp"
#include "iwp_matrix.hpp"

namespace iwp {

constexpr uint32_t NOBODY = 0xffffffffu;
// An expert's rows begin at a multiple of this, so that whole tiles of summed rows belong to one expert.
constexpr uint32_t PAD_ROWS = 64;

struct ExpertTile {
    uint32_t expert, first;                // first: of the expert's rows
};
struct ExpertRows {        // experts' rows after each other, in the order of slots; then the slots that nobody got
    uint32_t* start;       // [experts + 1]
    uint32_t* count;       // [experts + 1]
    uint32_t* slot;        // [padded rows] which slot a row is, NOBODY behind an expert's rows
    ExpertTile* tile;      // the experts' rows in tiles
    uint32_t* tiles;       // [2]: of the experts, of nobody
    uint32_t* counts;      // [workgroups that arrange, experts + 1]: slots of each one's part
};

// ------------------------------------------------------------------ the rows

// Which of the wavefront's lanes have the same value below 2048; those of `in` alone.
__device__ __forceinline__ uint64_t same_lanes(uint32_t value, bool in) {
    uint64_t same = __ballot(in);
#pragma unroll
    for (int bit = 0; bit < 11; ++bit) {
        const bool one = value >> bit & 1;
        const uint64_t ones = __ballot(one);
        same &= one ? ones : ~ones;
    }
    return same;
}

// Which slots go where.  Every workgroup has a part of the slots, every wavefront a part of that; slots of an expert stay in order.
constexpr uint32_t ARRANGE_WAVES = 16, ARRANGE_THREADS = ARRANGE_WAVES * 64;
struct SlotPart {
    uint32_t from, to;
    __device__ __forceinline__ SlotPart(uint32_t n, uint32_t per_wave) {
        const uint32_t wave = blockIdx.x * ARRANGE_WAVES + (threadIdx.x >> 6);
        from = min(wave * per_wave, n);
        to = min(from + per_wave, n);
    }
};
__device__ __forceinline__ uint32_t bucket_of(const int32_t* chosen, uint32_t i, uint32_t experts) { return min((uint32_t)chosen[i], experts); }

// Slots of every expert in each workgroup's part (where there is more than one).
__global__ void __launch_bounds__(ARRANGE_THREADS) k_expert_count(const int32_t* __restrict__ chosen, uint32_t n, uint32_t per_wave, uint32_t experts,
                                                                  ExpertRows R) {
    __shared__ uint32_t of[IWP_MAX_EXPERTS + 1];
    for (uint32_t e = threadIdx.x; e <= experts; e += ARRANGE_THREADS) of[e] = 0;
    __syncthreads();
    const SlotPart part(n, per_wave);
    for (uint32_t i = part.from + (threadIdx.x & 63); i < part.to; i += 64) atomicAdd(&of[bucket_of(chosen, i, experts)], 1u);
    __syncthreads();
    for (uint32_t e = threadIdx.x; e <= experts; e += ARRANGE_THREADS) R.counts[blockIdx.x * (experts + 1) + e] = of[e];
}

// Counts the wavefronts' parts, finds where the experts' rows begin and puts every slot in its place.  Every workgroup adds up the others'
// counts itself; the first one writes what is one for all.  Bound by its steps after each other: the slots' loads, counting, sums over wavefronts, another
// round for the places.  us for 32768 slots, 64 experts: one workgroup alone 52, counting and arranging by 32 of them 17.
__device__ __forceinline__ void arrange_slots(const int32_t* __restrict__ chosen, uint32_t n, uint32_t per_wave, uint32_t experts, uint32_t height,
                                              uint32_t workgroups, const ExpertRows& R) {
    __shared__ uint32_t at[ARRANGE_WAVES][IWP_MAX_EXPERTS + 1];
    __shared__ uint32_t rows_of[ARRANGE_WAVES], tiles_of[ARRANGE_WAVES], nobody_of[2];
    const uint32_t thread = threadIdx.x, wave = thread >> 6, lane = thread & 63;
    const SlotPart part(n, per_wave);
    for (uint32_t e = lane; e <= experts; e += 64) at[wave][e] = 0;
    lanes_exchange();
    for (uint32_t i = part.from + lane; i < part.to; i += 64) atomicAdd(&at[wave][bucket_of(chosen, i, experts)], 1u);
    __syncthreads();
    // slots of this thread's expert (the thread after the experts': nobody's) in all parts and in those before this workgroup's
    auto count = [&](uint32_t e, uint32_t* all, uint32_t* before) {
        *all = *before = 0;
        if (workgroups == 1) {
            for (uint32_t w = 0; w < ARRANGE_WAVES; ++w) *all += at[w][e];
            return;
        }
#pragma unroll 8
        for (uint32_t b = 0; b < workgroups; ++b) {
            const uint32_t c = R.counts[b * (experts + 1) + e];
            *all += c;
            if (b < blockIdx.x) *before += c;
        }
    };
    uint32_t mine = 0, before = 0, none = 0, none_before = 0;
    if (thread < experts) count(thread, &mine, &before);
    if (thread == ARRANGE_THREADS - 1) {
        count(experts, &none, &none_before);
        nobody_of[0] = none;
        nobody_of[1] = none_before;
    }
    const uint32_t padded = (mine + PAD_ROWS - 1) / PAD_ROWS * PAD_ROWS, tiles = (mine + height - 1) / height;
    uint32_t rows_to = padded, tiles_to = tiles;
    for (uint32_t o = 1; o < 64; o <<= 1) {
        const uint32_t a = __shfl_up(rows_to, o), b = __shfl_up(tiles_to, o);
        if (lane >= o) rows_to += a, tiles_to += b;
    }
    if (lane == 63) rows_of[wave] = rows_to, tiles_of[wave] = tiles_to;
    __syncthreads();
    uint32_t all_rows = 0, all_tiles = 0;
    for (uint32_t w = 0; w < ARRANGE_WAVES; ++w) {
        if (w < wave) rows_to += rows_of[w], tiles_to += tiles_of[w];
        all_rows += rows_of[w];
        all_tiles += tiles_of[w];
    }
    none = nobody_of[0];
    // what this thread's expert has, from `start` on
    auto put = [&](uint32_t e, uint32_t start, uint32_t count, uint32_t first_tile, uint32_t before) {
        if (blockIdx.x == 0) {
            R.start[e] = start;
            R.count[e] = count;
            for (uint32_t t = 0; e < experts && t * height < count; ++t) R.tile[first_tile + t] = ExpertTile{e, t * height};
        }
        uint32_t to = start + before;
        for (uint32_t w = 0; w < ARRANGE_WAVES; ++w) {
            const uint32_t c = at[w][e];
            at[w][e] = to;
            to += c;
        }
    };
    if (thread < experts) {
        const uint32_t start = rows_to - padded;
        put(thread, start, mine, tiles_to - tiles, before);
        if (blockIdx.x == 0)
            for (uint32_t r = start + mine; r < start + padded; ++r) R.slot[r] = NOBODY;
    }
    if (thread == 0) {
        put(experts, all_rows, none, all_tiles, nobody_of[1]);
        if (blockIdx.x == 0) R.tiles[0] = all_tiles, R.tiles[1] = (none + height - 1) / height;
    }
    __syncthreads();
    for (uint32_t base = part.from; base < part.to; base += 64) {
        const uint32_t i = base + lane;
        const bool in = i < part.to;
        const uint32_t e = in ? bucket_of(chosen, i, experts) : 0;
        const uint64_t same = same_lanes(e, in);
        const uint32_t rank = __popcll(same & ((1ull << lane) - 1)), first = at[wave][e];
        lanes_exchange();
        if (in) {
            R.slot[first + rank] = i;
            if (rank == 0) at[wave][e] = first + __popcll(same);
        }
        lanes_exchange();
    }
}

// 16 bytes of a row from element c on: zeros past its width
template <int SIZE>
__device__ __forceinline__ words4 row_chunk(const char* row, uint32_t c, uint32_t dim) {
    constexpr uint32_t CHUNK = 16 / SIZE;
    const char* p = row + (size_t)c * SIZE;
    if (c + CHUNK <= dim) return SIZE == 4 ? *reinterpret_cast<const words4*>(p) : (words4)*reinterpret_cast<const words4_any*>(p);
    words4 v = {};
#pragma unroll
    for (uint32_t e = 0; e < CHUNK; ++e)
        if (c + e < dim) {
            if (SIZE == 4) v[e % 4] = reinterpret_cast<const uint32_t*>(p)[e];
            else v[e / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[e] << (e % 2 * 16);
        }
    return v;
}

// How 16-byte units of a matrix's rows lie over workgroups: `units` to a row, threads over them all, GATHER_ROWS rows a thread.
constexpr uint32_t GATHER_ROWS = 4;
struct Units {
    uint32_t units, rows;
    __host__ __device__ uint32_t threads() const { return units * ((rows + GATHER_ROWS - 1) / GATHER_ROWS); }      // (launches_fit)
    __device__ __forceinline__ uint32_t unit(uint32_t thread) const { return thread % units; }
    __device__ __forceinline__ uint32_t row(uint32_t thread) const { return thread / units * GATHER_ROWS; }
};

// Matrices whose rows cannot be read by 16 bytes where they lie, into rows of whole units, zeros past the width.
struct MatrixCopy {
    const char* w;
    int64_t ld, step;
    uint32_t rows, columns;                // of a matrix
    Units of;                              // of all of them
    char* out;
};
template <int SIZE>
__device__ __forceinline__ void copy_matrices(const MatrixCopy& m, uint32_t thread) {
    constexpr uint32_t CHUNK = 16 / SIZE;
    const uint32_t u = m.of.unit(thread), r0 = m.of.row(thread);
    words4 v[GATHER_ROWS];
#pragma unroll
    for (uint32_t i = 0; i < GATHER_ROWS; ++i) {
        const uint32_t r = min(r0 + i, m.of.rows - 1), e = r / m.rows;
        v[i] = row_chunk<SIZE>(m.w + (e * m.step + (r - e * m.rows) * m.ld) * SIZE, u * CHUNK, m.columns);
    }
#pragma unroll
    for (uint32_t i = 0; i < GATHER_ROWS; ++i)
        if (r0 + i < m.of.rows) *reinterpret_cast<words4*>(m.out + ((size_t)(r0 + i) * m.of.units + u) * 16) = v[i];
}

// The first `arrangers` workgroups arrange the slots, the others copy matrices and rows that cannot be read where they lie, which does not
// wait for that.
template <int SIZE>
__global__ void __launch_bounds__(ARRANGE_THREADS) k_expert_arrange(const int32_t* __restrict__ chosen, uint32_t n, uint32_t per_wave, uint32_t experts,
                                                                    uint32_t height, uint32_t arrangers, ExpertRows R, MatrixCopy A, MatrixCopy B) {
    if (blockIdx.x < arrangers) {
        arrange_slots(chosen, n, per_wave, experts, height, arrangers, R);
        return;
    }
    const uint32_t thread = (blockIdx.x - arrangers) * ARRANGE_THREADS + threadIdx.x, first = A.of.threads();
    if (thread < first) copy_matrices<SIZE>(A, thread);
    else if (thread - first < B.of.threads()) copy_matrices<SIZE>(B, thread - first);
}

// Rows of a caller's matrix in the experts' order, zeros behind an expert's rows and past the width.  slots: of a token, whose row each of
// them has; 1: every slot has its own.
struct RowsGather {
    const char* x;
    int64_t ld;
    uint32_t dim, slots;
    Units of;
    char* out;
};
template <int SIZE>
__device__ __forceinline__ void gather_rows(const RowsGather& g, const ExpertRows& R, uint32_t rows, uint32_t thread) {
    constexpr uint32_t CHUNK = 16 / SIZE;
    const uint32_t u = g.of.unit(thread), r0 = g.of.row(thread);
    words4 v[GATHER_ROWS];
#pragma unroll
    for (uint32_t i = 0; i < GATHER_ROWS; ++i) {
        v[i] = words4{};
        const uint32_t slot = r0 + i < rows ? R.slot[r0 + i] : NOBODY;
        if (slot != NOBODY) v[i] = row_chunk<SIZE>(g.x + (int64_t)(g.slots == 1 ? slot : slot / g.slots) * g.ld * SIZE, u * CHUNK, g.dim);
    }
#pragma unroll
    for (uint32_t i = 0; i < GATHER_ROWS; ++i)
        if (r0 + i < rows) *reinterpret_cast<words4*>(g.out + ((size_t)(r0 + i) * g.of.units + u) * 16) = v[i];
}
// Two matrices' rows (the second's units may be none): the first `first` workgroups the first's.  32768 rows of 2048 and of 1024 elements in bf16, 64
// experts, 400 MB read and written: 62 us.  Four rows a thread: with eight 136 us for both.
template <int SIZE>
__global__ void __launch_bounds__(256) k_expert_gather(RowsGather A, RowsGather B, uint32_t first, uint32_t experts, ExpertRows R) {
    const bool second = blockIdx.x >= first;
    const uint32_t thread = (second ? blockIdx.x - first : blockIdx.x) * 256 + threadIdx.x;
    if (thread < (second ? B : A).of.threads()) gather_rows<SIZE>(second ? B : A, R, R.start[experts], thread);
}

// ------------------------------------------------------------------ the products

struct Matrices {          // one for every expert
    const char* w;
    int64_t step;          // elements from one to the next
    uint32_t ld, rows, columns;
};
struct Packed {            // gathered rows, or where they lie: a slot's own, or its token's
    const char* x;
    uint32_t ld, dim;
    uint32_t slots;        // of a token whose row is read where it lies (1: a row for every slot); 0: gathered
};
struct SlotRows {
    static constexpr bool ANYWHERE = true;
    const uint32_t* slot;
    uint32_t slots;
    __device__ __forceinline__ uint32_t operator()(uint32_t q) const { return slots == 1 ? slot[q] : slot[q] / slots; }
};
struct RowsOut {
    char* y;
    int64_t ld;            // elements
};

// What all lanes have alike, in a scalar register.
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ const uint16_t* uniform(const char* p) {
    const uint64_t at = reinterpret_cast<uintptr_t>(p);
    return reinterpret_cast<const uint16_t*>((uint64_t)uniform((uint32_t)(at >> 32)) << 32 | uniform((uint32_t)at));
}

// Where block `block` of n stands in the work's order: every die has a stretch of it.
__device__ __forceinline__ uint32_t stretch_place(uint32_t block, uint32_t n) {
    const uint32_t per = n / 8, more = n % 8, die = block % 8;
    return die * per + min(die, more) + block / 8;
}

// A wavefront's part of a tile to memory: row(q) is where the row of entry q begins, or null.
// Past the caches' order of use, so that stores do not displace the operands of the next tiles.  us of a call by ordinary stores and by these, bf16: 16384
// rows of 8 x 2048 x 4096 and reading all of y 331 and 311, 32768 of them 607 and 578; 8192 rows of 64 x 1024 x 1024, both gradients 160 and 130, 32768
// of 64 x 2048 x 1024 and the norm of dw 628 and 609.
template <class M, int OUT, int BP, int WP, class F>
__device__ __forceinline__ void store_tile(const M& mm, char* lds, uint32_t p0, uint32_t columns, F row_of) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    typedef Rows32<OUT == OUT_F32 ? 4 : 2, BP / WP> Out;
    static_assert(M::WAVES * Out::BYTES <= M::LDS, "a wavefront's rows");
    char* mine = lds + wave * Out::BYTES;
    constexpr uint32_t SIZE = OUT == OUT_F32 ? 4 : 2;
    const uint32_t pw = p0 + M::p_of(wave), qw = M::q_of(wave);
#pragma unroll
    for (int b = 0; b < M::FQ; ++b) {
#pragma unroll
        for (int a = 0; a < M::FP; ++a)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                f32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = mm.acc[a][b][c * 4 + e];
                uint64_t four = 0;
                if (OUT != OUT_F32)
#pragma unroll
                    for (int e = 0; e < 4; ++e) four |= (uint64_t)(OUT == OUT_BF16 ? Bf16::bits(v[e]) : F16::bits(v[e])) << (16 * e);
                Out::put(mine, a * 32 + p_in_fragment(c * 4, lane), lane, OUT == OUT_F32 ? (const void*)&v : (const void*)&four);
            }
        Out::each(mine, lane, [&](uint32_t row, uint32_t p, quad v) {
            if (pw + p >= columns) return;
            char* to = row_of(qw + b * 32 + row);
            if (!to) return;
            to += (size_t)(pw + p) * SIZE;
            if (pw + p + Out::PER_CHUNK <= columns) {
                __builtin_nontemporal_store(words4_any{v.x, v.y, v.z, v.w}, reinterpret_cast<words4_any*>(to));
            } else {
                const uint32_t word[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int e = 0; e < Out::PER_CHUNK; ++e)
                    if (pw + p + e < columns) {
                        if (OUT == OUT_F32) reinterpret_cast<uint32_t*>(to)[e] = word[e];
                        else reinterpret_cast<uint16_t*>(to)[e] = (uint16_t)(word[e / 2] >> (16 * (e & 1)));
                    }
            }
        });
    }
}

// Every expert's rows times its matrix (TRANSPOSED: W, not W^T, as for the rows' gradient), to the slots' rows of the output.
// at: which of the np x nq tiles, in an order in which some dozens in a row share few rows and columns.
template <class E, int BP, int BQ, int WP, int WQ, int OUT, bool TRANSPOSED, bool GATHERED, int W_LANE = 16>
__device__ __forceinline__ void rows_tile(const Matrices& W, const Packed& X, const ExpertRows& R, const RowsOut& Y, uint32_t at, uint32_t np, uint32_t nq,
                                          char* lds, uint32_t down = 0) {
    typedef Product<E, BP, BQ, WP, WQ, TRANSPOSED, false, W_LANE> M;
    const uint32_t columns = TRANSPOSED ? W.columns : W.rows;
    constexpr uint32_t TALL = 8;
    const uint32_t group = at / (np * TALL), rest = at - group * np * TALL, tall = min(TALL, nq - group * TALL);
    const uint32_t tp = rest / tall;
    ExpertTile tile = R.tile[group * TALL + rest % tall];
    tile = ExpertTile{uniform(tile.expert), uniform(tile.first) + down};
    const uint32_t count = uniform(R.count[tile.expert]), start = uniform(R.start[tile.expert]);
    if (tile.first >= count) return;                       // (a lower part of the tile)
    const uint32_t summed = TRANSPOSED ? W.rows : W.columns, to = (summed + M::DEEP - 1) / M::DEEP * M::DEEP;
    const Operand P{uniform(W.w + tile.expert * W.step * E::SIZE), nullptr, W.ld, columns, summed};
    const Operand Q{uniform(GATHERED ? X.x + (size_t)start * X.ld * E::SIZE : X.x), nullptr, X.ld, count, to};
    M mm;
    if constexpr (GATHERED) mm.run(P, Q, tp * BP, tile.first, 0, to, lds);
    else mm.run(P, Q, tp * BP, tile.first, 0, to, lds, SlotRows{R.slot + start, X.slots});
    constexpr uint32_t SIZE = OUT == OUT_F32 ? 4 : 2;
    store_tile<M, OUT, BP, WP>(mm, lds, tp * BP, columns, [&](uint32_t q) -> char* {
        if (tile.first + q >= count) return nullptr;
        return Y.y + (int64_t)R.slot[start + tile.first + q] * Y.ld * SIZE;
    });
}
// Zeros for the slots of nobody, a tile of their rows and the output's columns.  They come after the experts' tiles, which all dies share: in one order
// with these, dies with nobody's stretch would have nothing to multiply (an eighth of 65536 slots given, 8 experts of 2048 x 1024, bf16: 219 us
// instead of 72).
template <int BP, int BQ, int THREADS, int OUT>
__device__ __forceinline__ void nobody_tile(const ExpertRows& R, uint32_t experts, const RowsOut& Y, uint32_t at, uint32_t np, uint32_t columns) {
    constexpr uint32_t SIZE = OUT == OUT_F32 ? 4 : 2, CHUNK = 16 / SIZE, CHUNKS = BP / CHUNK;
    const uint32_t count = R.count[experts], p0 = at % np * BP, first = at / np * BQ;
    const uint32_t* slot = R.slot + R.start[experts];
    for (uint32_t i = threadIdx.x; i < BQ * CHUNKS; i += THREADS) {
        const uint32_t row = first + i / CHUNKS, p = p0 + i % CHUNKS * CHUNK;
        if (row >= count || p >= columns) continue;
        const int64_t to = slot[row] * Y.ld + p;
        if (p + CHUNK <= columns) {
            *reinterpret_cast<words4_any*>(Y.y + to * SIZE) = words4_any{};
        } else {
            for (uint32_t e = 0; p + e < columns; ++e) put<OUT>(Y.y, to + e, 0.0f);
        }
    }
}
template <class E, int BP, int BQ, int WP, int WQ, int OUT, bool GATHERED, int W_LANE>
__global__ void __launch_bounds__(WP * WQ * 64) k_expert_rows(Matrices W, Packed X, ExpertRows R, uint32_t experts, RowsOut Y) {
    __shared__ __align__(1024) char lds[Product<E, BP, BQ, WP, WQ, false, false>::LDS];
    const uint32_t np = (W.rows + BP - 1) / BP, nq = uniform(R.tiles[0]), n = np * nq;
    uint32_t after = blockIdx.x - n;
    if constexpr (BQ == 256) {                             // large tiles fill a compute unit each
        TilePart part;
        uint32_t whole;
        if (part_of(blockIdx.x, n, &part, &whole)) {
            if (part.half) rows_tile<E, BP, BQ / 2, 4, 2, OUT, false, GATHERED, W_LANE>(W, X, R, Y, part.tile, np, nq, lds, (part.half - 1) * (BQ / 2));
            else rows_tile<E, BP, BQ, WP, WQ, OUT, false, GATHERED, W_LANE>(W, X, R, Y, stretch_place(part.tile, whole), np, nq, lds);
            return;
        }
        after -= n - whole;                                // a workgroup more for each that was halved
    } else if (blockIdx.x < n) {
        rows_tile<E, BP, BQ, WP, WQ, OUT, false, GATHERED, W_LANE>(W, X, R, Y, stretch_place(blockIdx.x, n), np, nq, lds);
        return;
    }
    if (after < np * uniform(R.tiles[1])) nobody_tile<BP, BQ, WP * WQ * 64, OUT>(R, experts, Y, after, np, W.rows);
}

// Products of few rows, in one launch, without arranging anything: a workgroup has 16 rows of an expert's matrix, each of its wavefronts a
// quarter of their width; it finds the expert's slots by itself and takes 16 of them at a time, so a matrix is read once as long as its
// expert has no more.  Loads go straight to registers, whatever rows' alignment, eight steps of 16 rows by 64 bytes on their way.
struct FewF32 {
    static constexpr int SIZE = 4;
    static __device__ __forceinline__ f32x4 mfma(words4 a, words4 b, f32x4 c) {
#pragma unroll
        for (int k = 0; k < 4; ++k) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[k]), __uint_as_float(b[k]), c, 0, 0, 0);
        return c;
    }
};
struct FewBf16 {
    static constexpr int SIZE = 2;
    static __device__ __forceinline__ f32x4 mfma(words4 a, words4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};
struct FewF16 {
    static constexpr int SIZE = 2;
    static __device__ __forceinline__ f32x4 mfma(words4 a, words4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
};

constexpr uint32_t FEW_SLOTS = 1024, FEW_ROWS = 16;
// by_slot: a workgroup for every slot and 16 rows, of which the first slot of an expert does them all; else one for every expert, and one for nobody.
template <class E, int OUT>
__global__ void __launch_bounds__(256) k_expert_few(Matrices W, Packed X, const int32_t* __restrict__ chosen, uint32_t n, uint32_t experts, bool by_slot,
                                                    RowsOut Y) {
    constexpr uint32_t CHUNK = 16 / E::SIZE, STEP = 4 * CHUNK;
    __shared__ uint32_t list[FEW_SLOTS], found;
    __shared__ float sums[4][FEW_ROWS][FEW_ROWS + 1];
    const uint32_t np = (W.rows + FEW_ROWS - 1) / FEW_ROWS, p0 = blockIdx.x % np * FEW_ROWS, which = blockIdx.x / np;
    const uint32_t thread = threadIdx.x, lane = thread & 63, wave = thread >> 6;
    const uint32_t expert = by_slot ? bucket_of(chosen, which, experts) : which;
    if (thread == 0) found = 0;
    __syncthreads();
    bool earlier = false;
    for (uint32_t i = thread; i < n; i += 256) {
        if (bucket_of(chosen, i, experts) != expert || (by_slot && expert == experts && i != which)) continue;
        earlier |= i < which;
        list[atomicAdd(&found, 1u)] = i;
    }
    if (__syncthreads_or(by_slot && earlier)) return;
    const uint32_t count = found;
    if (expert == experts) {
        for (uint32_t i = thread; i < count * FEW_ROWS; i += 256)
            if (p0 + i % FEW_ROWS < W.rows) put<OUT>(Y.y, (int64_t)list[i / FEW_ROWS] * Y.ld + p0 + i % FEW_ROWS, 0.0f);
        return;
    }
    const uint32_t steps = (W.columns + STEP - 1) / STEP, each = (steps + 3) / 4, from = min(wave * each, steps), to = min(from + each, steps);
    const uint32_t whole = min(to, max(from, W.columns / STEP));
    const char* w = W.w + (expert * W.step + (int64_t)min(p0 + (lane & 15), W.rows - 1) * W.ld) * E::SIZE;
    const uint32_t c0 = (lane >> 4) * CHUNK;
    for (uint32_t r0 = 0; r0 < count; r0 += FEW_ROWS) {
        const uint32_t slot = list[min(r0 + (lane & 15), count - 1)];
        const char* x = X.x + (int64_t)(X.slots == 1 ? slot : slot / X.slots) * X.ld * E::SIZE;
        f32x4 acc = {};
        constexpr uint32_t AHEAD = 8;
        uint32_t s = from;
        for (; s + AHEAD <= whole; s += AHEAD) {
            words4 a[AHEAD], b[AHEAD];
#pragma unroll
            for (uint32_t k = 0; k < AHEAD; ++k) a[k] = row_chunk<E::SIZE>(w, (s + k) * STEP + c0, ~0u);
#pragma unroll
            for (uint32_t k = 0; k < AHEAD; ++k) b[k] = row_chunk<E::SIZE>(x, (s + k) * STEP + c0, ~0u);
#pragma unroll
            for (uint32_t k = 0; k < AHEAD; ++k) acc = E::mfma(a[k], b[k], acc);
        }
        for (; s < to; ++s) acc = E::mfma(row_chunk<E::SIZE>(w, s * STEP + c0, W.columns), row_chunk<E::SIZE>(x, s * STEP + c0, W.columns), acc);
#pragma unroll
        for (int j = 0; j < 4; ++j) sums[wave][(lane >> 4) * 4 + j][lane & 15] = acc[j];
        __syncthreads();
        const uint32_t p = thread & 15, q = thread >> 4;
        if (p0 + p < W.rows && r0 + q < count)
            put<OUT>(Y.y, (int64_t)list[r0 + q] * Y.ld + p0 + p, (sums[0][p][q] + sums[1][p][q]) + (sums[2][p][q] + sums[3][p][q]));
        __syncthreads();
    }
}

// An expert's matrix's gradient: the sum over its rows of dy x^T.
struct MatricesOut {
    char* w;
    int64_t ld, step;
};
template <class E, int BP, int BQ, int WP, int WQ, int OUT>
__device__ __forceinline__ void matrix_tile(const Packed& X, const Packed& D, const ExpertRows& R, const MatricesOut& dw, uint32_t at, char* lds) {
    typedef Product<E, BP, BQ, WP, WQ, true, true> M;
    const uint32_t np = (X.dim + BP - 1) / BP, nq = (D.dim + BQ - 1) / BQ;
    const uint32_t expert = at / (np * nq), of = at - expert * np * nq;
    constexpr uint32_t TALL = 8;
    const uint32_t group = of / (np * TALL), rest = of - group * np * TALL, tall = min(TALL, nq - group * TALL);
    const uint32_t tp = rest / tall, tq = group * TALL + rest % tall;
    const uint32_t rows = uniform((R.count[expert] + PAD_ROWS - 1) / PAD_ROWS * PAD_ROWS), start = uniform(R.start[expert]);
    const Operand P{uniform(X.x + (size_t)start * X.ld * E::SIZE), nullptr, X.ld, X.dim, rows};
    const Operand Q{uniform(D.x + (size_t)start * D.ld * E::SIZE), nullptr, D.ld, D.dim, rows};
    M mm;
    mm.run(P, Q, tp * BP, tq * BQ, 0, rows, lds);
    constexpr uint32_t SIZE = OUT == OUT_F32 ? 4 : 2;
    char* mine = dw.w + (expert * dw.step + (int64_t)tq * BQ * dw.ld) * SIZE;
    store_tile<M, OUT, BP, WP>(mm, lds, tp * BP, X.dim, [&](uint32_t q) -> char* { return tq * BQ + q < D.dim ? mine + (int64_t)q * dw.ld * SIZE : nullptr; });
}

// Both gradients in one launch, eights of tiles of either in turn, so that tiles that write and tiles that multiply run at the same time.
// rows, nobodys, matrices: whether the rows' gradient is wanted, and zeros in nobody's; the tiles of the matrices'.  Experts have more and fewer rows, so the dies take the
// matrices' neighbouring tiles in turn: with a stretch of the experts each, the die with the liked ones is the last (8 experts of 2048 x 4096, 16384
// rows: 411 us instead of 275; 64 of 2048 x 1024, 65536 rows: 458 and 400).
template <class E, int BP, int BQ, int WP, int WQ, int OUT_X, int OUT_W, int W_LANE>
__global__ void __launch_bounds__(WP * WQ * 64) k_expert_gradients(Matrices W, Packed X, Packed D, ExpertRows R, uint32_t experts, RowsOut dx, bool rows,
                                                                   bool nobodys, MatricesOut dw, uint32_t matrices) {
    __shared__ __align__(1024) char lds[Product<E, BP, BQ, WP, WQ, true, true>::LDS];
    const uint32_t np = (W.columns + BP - 1) / BP, nq = rows ? uniform(R.tiles[0]) : 0;
    const uint32_t eights = (np * nq + 7) / 8, others = (matrices + 7) / 8, all = eights + others, i = blockIdx.x / 8, die = blockIdx.x % 8;
    if (i >= all) {
        const uint32_t after = (i - all) * 8 + die;
        if (nobodys && after < np * uniform(R.tiles[1])) nobody_tile<BP, BQ, WP * WQ * 64, OUT_X>(R, experts, dx, after, np, W.columns);
        return;
    }
    const uint32_t before = (uint32_t)((uint64_t)i * eights / all), after = (uint32_t)((uint64_t)(i + 1) * eights / all);
    if (after > before) {
        const uint32_t at = before * 8 + die;
        if (at < np * nq) rows_tile<E, BP, BQ, WP, WQ, OUT_X, true, true, W_LANE>(W, D, R, dx, stretch_place(at, np * nq), np, nq, lds);
    } else {
        const uint32_t at = (i - before) * 8 + die;
        if (at < matrices) matrix_tile<E, BP, BQ, WP, WQ, OUT_W>(X, D, R, dw, at, lds);
    }
}

// A token's gradient: the sum over its slots' rows, in their order.  Four entries a thread.
template <int OUT>
__global__ void __launch_bounds__(256) k_expert_sum(const float* __restrict__ rows, uint32_t ld, const int32_t* __restrict__ chosen, uint32_t tokens,
                                                    uint32_t slots, uint32_t experts, uint32_t dim, uint32_t first, Spread spread, void* __restrict__ dx,
                                                    int64_t ld_dx) {
    const uint32_t token = first + spread.row(), c = spread.unit() * 4;
    if (token >= tokens || c >= dim) return;
    f32x4 sum = {};
    for (uint32_t k = 0; k < slots; ++k) {
        const size_t slot = (size_t)token * slots + k;
        if ((uint32_t)chosen[slot] < experts) sum += *reinterpret_cast<const f32x4*>(rows + slot * ld + c);
    }
    const int64_t to = token * ld_dx + c;
    if (c + 4 <= dim && OUT == OUT_F32) {
        *reinterpret_cast<words4*>(static_cast<float*>(dx) + to) = __builtin_bit_cast(words4, sum);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c + e < dim) iwp::put<OUT>(dx, to + e, sum[e]);
    }
}

}  // namespace iwp
