// Matrix products on 16-bit operands (bf16, fp16) with binary32 sums, tiled for gfx950's matrix cores.  One tile loop for
// every product of the head kernels; what differs is which way an operand lies in memory:
//   rows of K     the summed index is contiguous; a lane's fragment is one 128-bit LDS read
//   columns of K  the other index is contiguous; a lane's fragment is two transposing 64-bit LDS reads
// The tile of P is the matrix instruction's first operand, that of Q its second, so a lane ends up with four consecutive
// entries of P for one entry of Q: P is the index that is contiguous in the product, Q its row.
//
// Bound by the matrix cores and the power that they draw.  8192 tokens x 4096 x 131072 entries in bf16, 8.8 TFLOP a product: logits
// with their statistics 7.0 to 7.4 ms (1.2 to 1.26 PFLOP/s), dH 6.8 to 7.3, dW 7.0 to 7.2 (1.2 to 1.3); the library's products of
// 8192^3 reach 1.40, 1.23 and 1.09 for the same three layouts.  The matrix cores are busy 63 to 67 % of the cycles, at a clock of
// 1.75 to 1.82 GHz instead of 2.4; LDS has no bank conflicts, and what is fetched from memory is 7 GB a product.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace iwp {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
// What is written to memory as one type and read as another goes through these: the compiler may not take such accesses apart by their type.
typedef uint32_t quad __attribute__((ext_vector_type(4), may_alias));
typedef float f32x4_bytes __attribute__((ext_vector_type(4), may_alias));
typedef float f32_bytes __attribute__((may_alias));
typedef uint64_t u64_bytes __attribute__((may_alias));

// Between writes to LDS and reads of them by other lanes of the same wavefront, in either order: no instruction (a wavefront's LDS accesses
// are done in order), but the compiler must not move them across.
__device__ __forceinline__ void lanes_exchange() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

struct Bf16 {
    static __device__ __forceinline__ f32x16 mfma(s16x8 a, s16x8 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint16_t bits(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
    static __device__ __forceinline__ float value(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }
};
struct F16 {
    static __device__ __forceinline__ f32x16 mfma(s16x8 a, s16x8 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint16_t bits(float x) { return __builtin_bit_cast(uint16_t, (_Float16)x); }
    static __device__ __forceinline__ float value(uint16_t b) { return (float)__builtin_bit_cast(_Float16, b); }
};

constexpr uint32_t BK = 64;                        // summed entries per LDS tile: 128 bytes of a row

// An operand as the tile loop reads it.  Binary32 operands come as two planes of fp16 (see split_f32): `lo` is null for
// operands of 16 bits.
struct Operand {
    const uint16_t* hi;
    const uint16_t* lo;
    uint32_t ld;           // elements from row to row; ld * 512 bytes stay below 2^32
    uint32_t extent;       // valid entries of the index that is not summed
    uint32_t summed;       // valid entries of the summed one
};

// 16 bytes per lane from `base` + the lane's offset straight to LDS, lane after lane from `lds` (uniform) on.  In assembly,
// because the compiler waits for such loads before any transposing read, of whichever tile; wait_for_loads() waits for them.
// (m0 is no register that the compiler keeps anything in: it sets it where an instruction of its own needs it.)
__device__ __forceinline__ void load_to_lds(const char* base, uint32_t offset, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(base), "s"(lds) : "memory");
}
// Until at most LEFT of this wavefront's loads are on their way and all of its LDS reads are done.
template <int LEFT>
__device__ __forceinline__ void wait_for_loads() {
    static_assert(LEFT < 64, "six bits");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(LEFT) : "memory");
}
__device__ __forceinline__ void workgroup_barrier() {
    asm volatile("s_barrier" ::: "memory");
}
__device__ __forceinline__ uint32_t lds_address(const void* p) {
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char*)p;
}

// One operand's tile: R entries of its own index, BK of the summed one, WAVES wavefronts loading.
//
// Rows of K: LDS row r holds the 8 chunks (16 bytes) of entry r, chunk c at place c ^ turn(r).
// Columns of K: LDS row k holds R entries, in pairs of chunks of 64 bytes, pair p at place p ^ turn.
// Both turns spread what one LDS access reads over the banks.  The loads go straight to LDS, lane by lane in address order, so
// it is the address in global memory that is turned.
//
// Entries past the operand's extent are read from a valid one: what they contribute to is never stored.  Summed entries past
// an operand's end are read from the same row, or from its last row; of the two operands one always reaches to a multiple of BK
// and holds zeros there.
template <int R, int WAVES, bool COLUMNS>
struct Tile {
    static constexpr int BYTES = R * BK * 2;
    static constexpr int LOADS = BYTES / 1024 / WAVES;      // 64 lanes of 16 bytes each
    static_assert(LOADS * WAVES * 1024 == BYTES, "whole loads");
    static constexpr int PER_ROW = COLUMNS ? R / 8 : BK / 8;
    static constexpr int TURNS = COLUMNS ? (R / 32 < 8 ? R / 32 : 8) : 8;

    uint32_t at[LOADS];        // byte offset of this lane's chunk from the tile's origin
    uint32_t within[LOADS];    // its (first) summed index in the tile
    uint32_t row_bytes;

    static __device__ __forceinline__ uint32_t turn(uint32_t r) {
        if (!COLUMNS) return (r >> 1) & 7u;
        return ((r & 3u) | ((r >> 1) & 4u)) & (TURNS - 1);
    }
    __device__ __forceinline__ void init(const Operand& o, uint32_t first, int wave, int lane) {
        row_bytes = o.ld * 2;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const uint32_t slot = (wave * LOADS + i) * 64 + lane, row = slot / PER_ROW, place = slot % PER_ROW;
            if (!COLUMNS) {
                const uint32_t entry = min(first + row, o.extent - 1) - first, chunk = place ^ turn(row);
                within[i] = chunk * 8;
                at[i] = entry * row_bytes + chunk * 16;
            } else {
                const uint32_t chunk = (((place >> 2) ^ turn(row)) << 2) | (place & 3u);
                const uint32_t entry = first + chunk * 8 < o.extent ? chunk * 8 : 0u;
                within[i] = row;
                at[i] = entry * 2 + row * row_bytes;
            }
        }
    }
    // plane + first entry, as bytes: where the tile's entry 0 at summed index k lies
    static __device__ __forceinline__ const char* origin(const uint16_t* plane, const Operand& o, uint32_t first, uint32_t k) {
        return reinterpret_cast<const char*>(plane) + (COLUMNS ? ((size_t)k * o.ld + first) * 2 : ((size_t)first * o.ld + k) * 2);
    }
    // The i-th load; left: summed entries from the tile's first on (at least 1)
    __device__ __forceinline__ void load(int i, const char* from, uint32_t left, uint32_t lds, int wave) const {
        const uint32_t inside = COLUMNS ? at[i] - (within[i] - (left - 1)) * row_bytes : at[i] - within[i] * 2;
        load_to_lds(from, within[i] < left ? at[i] : inside, lds + (wave * LOADS + i) * 1024);
    }
    // Fragment of the 32 entries from `entry` (a multiple of 32) on, summed indices 16 s to 16 s + 15 of the tile.
    static __device__ __forceinline__ s16x8 fragment(const char* lds, uint32_t entry, int s, int lane) {
        if (!COLUMNS) {
            const uint32_t row = entry + (lane & 31), chunk = 2 * s + (lane >> 5);
            return *reinterpret_cast<const s16x8*>(lds + row * (BK * 2) + ((chunk ^ turn(row)) << 4));
        }
        const uint32_t i = lane & 15, half = lane >> 5;
        const uint32_t k = 16 * s + 8 * half + (i >> 2);
        const char* p = lds + k * (R * 2) + (((entry >> 5) ^ turn(k)) << 6) + ((lane >> 4) & 1) * 32 + (i & 3) * 8;
        typedef __attribute__((address_space(3))) s16x4* lds_quad;
        const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_quad)p);
        const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_quad)(p + 4 * R * 2));
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
};

// The product of a BP x BQ tile: WP x WQ wavefronts, each BP / WP entries of P by BQ / WQ of Q.
//
// 256 x 256 with 8 wavefronts of 128 x 64 each takes 128 accumulators a lane, two wavefronts a SIMD, and 128 of the 160 KB of LDS for
// two tiles.  ms for the logits, dH and dW of the size above: fragments read where they are needed 8.6, 9.6, 12.0; a step ahead,
// and with the tile's loads in flight for a whole tile 8.0, 7.3, 9.5; outputs through LDS (Rows32) 7.8, 7.5, 7.6; reads and loads
// one by one between the matrix instructions 7.55, 7.3, 7.15; priority to the wavefronts that issue loads, 1 to 2 % less.  Four
// tiles of 32 summed entries instead of two of 64: 8.3, 8.3, 8.15 against 7.8, 7.5, 7.6 (a barrier twice as often costs more than the
// longer flight of the loads gains).  Wavefronts of 256 x 32, which read half as much LDS again: dH 8.0 to 8.1 against 7.2 to
// 7.3; of 64 x 128: the same within 1 %.
template <class E, int BP, int BQ, int WP, int WQ, bool P_COLUMNS, bool Q_COLUMNS>
struct Product {
    static constexpr int WAVES = WP * WQ;
    static constexpr int FP = BP / WP / 32, FQ = BQ / WQ / 32;     // fragments of 32 per wavefront
    typedef Tile<BP, WAVES, P_COLUMNS> TP;
    typedef Tile<BQ, WAVES, Q_COLUMNS> TQ;
    static constexpr int STAGE = TP::BYTES + TQ::BYTES, LDS = 2 * STAGE;

    f32x16 acc[FP][FQ];

    // entries of P and Q of this wavefront inside the tile, and of register r of a fragment inside it
    static __device__ __forceinline__ uint32_t p_of(int wave) { return (wave % WP) * (BP / WP); }
    static __device__ __forceinline__ uint32_t q_of(int wave) { return (wave / WP) * (BQ / WQ); }

    // Sum over summed indices [k_from, k_to), a multiple of BK, of P[p0 ..][k] Q[q0 ..][k].  Operands of two planes x = hi + 2^-11 lo (scaled, see
    // split_f32) take three passes, lo hi + hi lo first, then times 2^-11, then hi hi; lo lo lies below binary32.
    __device__ __forceinline__ void run(const Operand& P, const Operand& Q, uint32_t p0, uint32_t q0, uint32_t k_from,
                                        uint32_t k_to, char* lds) {
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
        for (int a = 0; a < FP; ++a)
#pragma unroll
            for (int b = 0; b < FQ; ++b) acc[a][b] = f32x16{};
        if (k_from >= k_to) return;
        TP tp;
        TQ tq;
        tp.init(P, p0, wave, lane);
        tq.init(Q, q0, wave, lane);
        const uint32_t steps = (k_to - k_from) / BK, passes = P.lo ? 3 : 1, total = steps * passes;
        const uint32_t pw = p_of(wave), qw = q_of(wave);
        const size_t p_step = (P_COLUMNS ? (size_t)P.ld * BK : BK) * 2, q_step = (Q_COLUMNS ? (size_t)Q.ld * BK : BK) * 2;
        const char *pf = nullptr, *qf = nullptr;
        uint32_t step = 0, pass = 0;                                   // of the next tile to be loaded
        const uint32_t lds_at = lds_address(lds);
        constexpr int LOADS = TP::LOADS + TQ::LOADS, STEPS = BK / 16, PRODUCTS = FP * FQ;
        // load i of the tile `step` of `pass`, into a stage; advance() goes on to the next tile
        auto origin = [&]() {
            pf = TP::origin(passes == 3 && pass == 0 ? P.lo : P.hi, P, p0, k_from);
            qf = TQ::origin(passes == 3 && pass == 1 ? Q.lo : Q.hi, Q, q0, k_from);
        };
        auto load = [&](int i, uint32_t stage) {
            const uint32_t k = k_from + step * BK, to = lds_at + stage * STAGE;
            if (i < TP::LOADS) tp.load(i, pf, P.summed - k, to, wave);
            else tq.load(i - TP::LOADS, qf, Q.summed - k, to + TP::BYTES, wave);
        };
        auto advance = [&]() {
            pf += p_step;
            qf += q_step;
            if (++step == steps) {
                step = 0;
                ++pass;
                origin();
            }
        };
        origin();
        s16x8 fp[2][FP], fq[2][FQ];
        auto read = [&](int i, uint32_t stage, int s, int to) {        // fragment i of a step
            const char* lp = lds + stage * STAGE;
            if (i < FQ) fq[to][i] = TQ::fragment(lp + TP::BYTES, qw + i * 32, s, lane);
            else fp[to][i - FQ] = TP::fragment(lp, pw + (i - FQ) * 32, s, lane);
        };
        // One tile.  Fragments are read a step of 16 ahead of the matrix instructions that take them, the first of a tile during the
        // last step of the tile before.  At that point every wavefront has read all it needs of the old tile, whose place the loads
        // of the tile after the next then take: they have a whole tile's products to arrive in.  Reads and loads go out one
        // by one between the matrix instructions; left to itself the compiler puts them in front of these, in bursts.
        auto tile = [&](auto next, auto more, uint32_t stage) {
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                const bool last = s + 1 == STEPS;
                if (last && next) {
                    wait_for_loads<0>();
                    workgroup_barrier();
                    __builtin_amdgcn_s_setprio(1);                     // the wavefront whose loads are due goes first
                }
                if (s == 0) __builtin_amdgcn_s_setprio(0);
#pragma unroll
                for (int i = 0; i < PRODUCTS; ++i) {
#pragma unroll
                    for (int r = i; r < FP + FQ; r += PRODUCTS) {
                        if (!last) read(r, stage, s + 1, (s + 1) & 1);
                        else if (next) read(r, stage ^ 1, 0, 0);
                    }
                    if (last && more)
#pragma unroll
                        for (int l = i; l < LOADS; l += PRODUCTS) load(l, stage);
                    acc[i / FQ][i % FQ] = E::mfma(fp[s & 1][i / FQ], fq[s & 1][i % FQ], acc[i / FQ][i % FQ]);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            if (more) advance();
        };
        constexpr std::true_type yes{};
        constexpr std::false_type no{};
#pragma unroll
        for (int i = 0; i < LOADS; ++i) load(i, 0);
        advance();
        if (total > 1) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) load(i, 1);
            advance();
            wait_for_loads<LOADS>();
        } else {
            wait_for_loads<0>();
        }
        workgroup_barrier();
#pragma unroll
        for (int i = 0; i < FP + FQ; ++i) read(i, 0, 0, 0);
        uint32_t t = 0;
        auto rescale = [&]() {
            if (passes == 3 && t == 2 * steps) {
#pragma unroll
                for (int a = 0; a < FP; ++a)
#pragma unroll
                    for (int b = 0; b < FQ; ++b) acc[a][b] *= 0x1p-11f;
            }
        };
        for (; t + 2 < total; ++t) {
            rescale();
            tile(yes, yes, t & 1);
        }
        if (t + 1 < total) {
            rescale();
            tile(yes, no, t & 1);
            ++t;
        }
        rescale();
        tile(no, no, t & 1);
        __syncthreads();                                               // the LDS is free for what follows
    }
};

// Register r of a fragment: entry of P inside the fragment's 32 (the entry of Q is lane & 31).
__device__ __forceinline__ uint32_t p_in_fragment(int r, int lane) { return 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3); }

// A wavefront's way from accumulators to memory: 32 rows (entries of Q) of its entries of P, through LDS, so that a store instruction
// writes whole stretches of rows.  As the matrix instructions leave them, a lane holds four entries of a row and neighbouring
// lanes neighbouring rows.  Chunks of 16 bytes are turned by the row, which keeps both sides off each other's banks.
template <int SIZE, int ENTRIES>                   // bytes per entry: 2 or 4
struct Rows32 {
    static constexpr int CHUNKS = ENTRIES * SIZE / 16, BYTES = 32 * ENTRIES * SIZE, PER_CHUNK = 16 / SIZE;
    static constexpr uint32_t TURNS = CHUNKS < 16 ? CHUNKS : 16;
    static __device__ __forceinline__ uint32_t place(uint32_t row, uint32_t chunk) {
        return (row * CHUNKS + (chunk ^ (row & (TURNS - 1)))) * 16;
    }
    // four entries from p on (a multiple of 4) of this lane's row
    static __device__ __forceinline__ void put(char* lds, uint32_t p, int lane, const void* four) {
        char* to = lds + place(lane & 31, p / PER_CHUNK) + (p % PER_CHUNK) * SIZE;
        if (SIZE == 2) *reinterpret_cast<u64_bytes*>(to) = *static_cast<const u64_bytes*>(four);
        else *reinterpret_cast<f32x4_bytes*>(to) = *static_cast<const f32x4_bytes*>(four);
    }
    static __device__ __forceinline__ float value(const char* lds, uint32_t row, uint32_t p) {      // of 4 bytes
        return *reinterpret_cast<const f32_bytes*>(lds + place(row, p / 4) + (p % 4) * 4);
    }
    // store(row, first entry, 16 bytes) for every chunk
    template <class F>
    static __device__ __forceinline__ void each(const char* lds, int lane, F store) {
        lanes_exchange();
#pragma unroll
        for (int i = 0; i < 32 * CHUNKS / 64; ++i) {
            const uint32_t at = i * 64 + lane, row = at / CHUNKS, chunk = at % CHUNKS;
            store(row, chunk * PER_CHUNK, *reinterpret_cast<const quad*>(lds + place(row, chunk)));
        }
        lanes_exchange();
    }
};

}  // namespace iwp
