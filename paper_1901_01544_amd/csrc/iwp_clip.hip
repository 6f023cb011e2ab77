// Clipping of the workers' gradients (include/iwp_clip.h): kernels and host side.
//
// Bound by memory: a gradient is read for its norm and read again to be scaled and written, 12 bytes an element where 8 cannot be
// done without; what the memory-side cache still has of it is not read twice (see LONG_BYTES).  A wavefront takes a chunk of 2048 elements at a
// time, eight loads of 16 bytes a lane on their way.  Squares are exact in binary64, sums in a fixed order: lane, wavefront, workgroup,
// then the worker's workgroups.  8 workers of 61 M elements: 935 us, 6.3 TB/s of 12 bytes an element; norms alone 323 us, 6.0 TB/s.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "../../include/iwp_clip.h"
#include "iwp_host.hpp"

using namespace iwp;

namespace {

typedef uint32_t words4 __attribute__((ext_vector_type(4), aligned(4), may_alias));

constexpr uint32_t CHUNK = 2048, LOADS = CHUNK / 256;

struct TensorChunk {
    uint64_t offset;
    uint32_t n, pad;
};

struct ClipCall {
    const TensorChunk* chunks;
    uint32_t n_chunks, blocks;             // workgroups of a worker
    double scale, max_norm;
    float* norm;
    double* sums;                          // [W, blocks]
    const float* g[IWP_MAX_WORKERS];
    float* out[IWP_MAX_WORKERS];
};

__device__ __forceinline__ double wave_sum(double s) {
    for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
    return s;
}

// A chunk's elements of this lane; zeros past its end.  LAST_USE: the caches need not keep them.
template <bool LAST_USE>
__device__ __forceinline__ void load_chunk(const float* from, uint32_t n, words4 (&v)[LOADS]) {
    const uint32_t lane = threadIdx.x & 63;
    if (n == CHUNK) {
#pragma unroll
        for (uint32_t j = 0; j < LOADS; ++j) {
            const words4* at = reinterpret_cast<const words4*>(from + (j * 64 + lane) * 4);
            v[j] = LAST_USE ? __builtin_nontemporal_load(at) : *at;
        }
        return;
    }
#pragma unroll
    for (uint32_t j = 0; j < LOADS; ++j) {
        const uint32_t e = (j * 64 + lane) * 4;
        v[j] = words4{};
        if (e + 4 <= n) v[j] = *reinterpret_cast<const words4*>(from + e);
        else
#pragma unroll
            for (uint32_t i = 0; i < 3; ++i)
                if (e + i < n) v[j][i] = __float_as_uint(from[e + i]);
    }
}
__device__ __forceinline__ void store_chunk(float* to, uint32_t n, const words4 (&v)[LOADS]) {
    const uint32_t lane = threadIdx.x & 63;
#pragma unroll
    for (uint32_t j = 0; j < LOADS; ++j) {
        const uint32_t e = (j * 64 + lane) * 4;
        if (e + 4 <= n) __builtin_nontemporal_store(v[j], reinterpret_cast<words4*>(to + e));
        else
#pragma unroll
            for (uint32_t i = 0; i < 3; ++i)
                if (e + i < n) to[e + i] = __uint_as_float(v[j][i]);
    }
}

// Sum of the squares of the chunks that wavefront `wave` of `waves` takes, in every lane.
__device__ __forceinline__ double squares(const ClipCall& c, const float* g, uint32_t wave, uint32_t waves) {
    double sum[4] = {};
    for (uint32_t k = wave; k < c.n_chunks; k += waves) {
        const TensorChunk at = c.chunks[k];
        words4 v[LOADS];
        load_chunk<false>(g + at.offset, at.n, v);
#pragma unroll
        for (uint32_t j = 0; j < LOADS; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const double x = (double)__uint_as_float(v[j][i]);
                sum[i] = __builtin_fma(x, x, sum[i]);
            }
    }
    return wave_sum((sum[0] + sum[1]) + (sum[2] + sum[3]));
}

// The sum of all wavefronts' values, in every thread.
template <int WAVES>
__device__ __forceinline__ double workgroup_sum(double s) {
    __shared__ double of[WAVES];
    __syncthreads();
    if ((threadIdx.x & 63) == 0) of[threadIdx.x >> 6] = s;
    __syncthreads();
    double all = of[0];
    for (int v = 1; v < WAVES; ++v) all += of[v];
    return all;
}

// What a gradient is multiplied by; its norm.  Where it is clipped, the scale is left out of quotient and product alike: the norm with it may lie above
// binary64.
__device__ __forceinline__ double factor(const ClipCall& c, double square, float* norm) {
    const double root = sqrt(square), n = fabs(c.scale) * root;
    *norm = (float)n;
    return n <= c.max_norm ? c.scale : copysign(c.max_norm / root, c.scale);
}

// A wavefront's chunks of a product.  The last chunks first: they are what the memory-side cache still has of the pass for the norm.  The first
// one is requested before the factor is known, unless a gradient may stay as it is.  (8 workers of 61 M elements in place and not clipped: 389 us, with
// that request 449.)
template <bool LAST_USE>
struct Multiplier {
    const ClipCall& c;
    const float* g;
    float* out;
    uint32_t wave, waves;
    TensorChunk at;
    words4 v[LOADS];
    __device__ __forceinline__ void request(uint32_t k) {
        at = c.chunks[c.n_chunks - 1 - k];
        load_chunk<LAST_USE>(g + at.offset, at.n, v);
    }
    __device__ __forceinline__ Multiplier(const ClipCall& c, uint32_t p, uint32_t wave, uint32_t waves) : c(c), g(c.g[p]), out(c.out[p]), wave(wave), waves(waves) {
        if (out && out != g && wave < c.n_chunks) request(wave);
    }
    __device__ __forceinline__ void by(double factor) {
        if (!out || (factor == 1.0 && out == g)) return;
        if (out == g && wave < c.n_chunks) request(wave);
        for (uint32_t k = wave; k < c.n_chunks;) {
#pragma unroll
            for (uint32_t j = 0; j < LOADS; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) v[j][i] = __float_as_uint((float)((double)__uint_as_float(v[j][i]) * factor));
            store_chunk(out + at.offset, at.n, v);
            k += waves;
            if (k < c.n_chunks) request(k);
        }
    }
};

__global__ void __launch_bounds__(256) k_clip_norm(ClipCall c, uint32_t first) {
    const uint32_t p = first + blockIdx.x / c.blocks, block = blockIdx.x % c.blocks;
    if (!c.g[p]) return;
    const double s = workgroup_sum<4>(squares(c, c.g[p], block * 4 + (threadIdx.x >> 6), c.blocks * 4));
    if (threadIdx.x == 0) c.sums[(size_t)p * c.blocks + block] = s;
}

// Every workgroup joins its worker's sums; the worker's first one has the norm.  Without an out, there is one workgroup a worker.
template <bool LAST_USE>
__global__ void __launch_bounds__(256) k_clip_apply(ClipCall c, uint32_t first, uint32_t blocks) {
    const uint32_t p = first + blockIdx.x / blocks, block = blockIdx.x % blocks;
    if (!c.g[p]) {
        if (block == 0 && threadIdx.x == 0) c.norm[p] = 0.0f;
        return;
    }
    Multiplier<LAST_USE> m(c, p, block * 4 + (threadIdx.x >> 6), blocks * 4);
    double s = 0.0;
    for (uint32_t b = threadIdx.x; b < c.blocks; b += 256) s += c.sums[(size_t)p * c.blocks + b];
    s = workgroup_sum<4>(wave_sum(s));
    float norm;
    const double by = factor(c, s, &norm);
    if (block == 0 && threadIdx.x == 0) c.norm[p] = norm;
    m.by(by);
}

// All of a worker in one workgroup, for small tables.
__global__ void __launch_bounds__(1024) k_clip_one(ClipCall c) {
    const uint32_t p = blockIdx.x, wave = threadIdx.x >> 6;
    if (!c.g[p]) {
        if (threadIdx.x == 0) c.norm[p] = 0.0f;
        return;
    }
    float norm;
    const double by = factor(c, workgroup_sum<16>(squares(c, c.g[p], wave, 16)), &norm);
    if (threadIdx.x == 0) c.norm[p] = norm;
    Multiplier<false>(c, p, wave, 16).by(by);
}

constexpr uint32_t GRID = 2048;            // 256 threads each: what the compute units hold at a time
constexpr uint32_t ONE_CHUNKS = 64;        // four a wavefront of the one workgroup

// Where the memory-side cache (256 MiB) ends.  us for 8 workers of 61 M elements: norms and products of all workers after each other 1084; what
// is written past the cache 1065, what is read last too 996; a worker at a time, whose gradient the cache then has part of, 935.  8 x 25 M:
// all after each other, past the cache, 380, in fours 410.  8 x 8 M, which the cache holds: 115, reading past it 120.  Norms alone of 8 x 61 M: 323,
// a worker at a time 372.
constexpr uint64_t CACHE_BYTES = 256ull << 20, LONG_BYTES = 160ull << 20;
uint64_t worker_bytes(uint32_t n_chunks) { return (uint64_t)n_chunks * CHUNK * sizeof(float); }
uint32_t at_a_time(uint32_t n_chunks, uint32_t W) { return worker_bytes(n_chunks) > LONG_BYTES ? 1 : W; }
uint32_t blocks_of(uint32_t n_chunks, uint32_t W) { return std::max(1u, std::min((n_chunks + 3) / 4, GRID / at_a_time(n_chunks, W))); }

inline bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

}  // namespace

struct iwp_tensors {
    TensorChunk* chunks = nullptr;         // on the device
    uint32_t n_chunks = 0;
    uint64_t begin = 0, end = 0;           // of the elements
};

extern "C" {

int iwp_tensors_create(const iwp_layer* rows, uint32_t n_rows, iwp_tensors** tensors_out) {
    if (!tensors_out) return IWP_EINVAL;
    *tensors_out = nullptr;
    if (!rows || n_rows == 0) return IWP_EINVAL;
    uint64_t end = 0, n_chunks = 0;
    for (uint32_t j = 0; j < n_rows; ++j) {
        if (rows[j].offset < 0 || (uint64_t)rows[j].offset < end) return IWP_EINVAL;           // table order, no overlap
        end = (uint64_t)rows[j].offset + rows[j].n;
        if (end > IWP_MAX_FLAT) return IWP_ERANGE;
        n_chunks += (rows[j].n + (uint64_t)CHUNK - 1) / CHUNK;
    }
    std::vector<TensorChunk> chunks;
    iwp_tensors* t = new (std::nothrow) iwp_tensors;
    try {
        chunks.reserve(std::max<uint64_t>(n_chunks, 1));
    } catch (...) {
        delete t;
        t = nullptr;
    }
    if (!t) return hip_fail(hipErrorOutOfMemory, "iwp_tensors_create");
    t->begin = end;
    for (uint32_t j = 0; j < n_rows; ++j)
        for (uint64_t at = 0; at < rows[j].n; at += CHUNK) {
            t->begin = std::min(t->begin, (uint64_t)rows[j].offset);
            chunks.push_back(TensorChunk{(uint64_t)rows[j].offset + at, (uint32_t)std::min<uint64_t>(CHUNK, rows[j].n - at), 0});
        }
    t->n_chunks = (uint32_t)chunks.size();
    t->end = chunks.empty() ? t->begin : chunks.back().offset + chunks.back().n;
    const size_t bytes = std::max<size_t>(1, chunks.size()) * sizeof(TensorChunk);
    hipError_t e = hipMalloc(reinterpret_cast<void**>(&t->chunks), bytes);
    if (e == hipSuccess && !chunks.empty()) e = hipMemcpy(t->chunks, chunks.data(), bytes, hipMemcpyHostToDevice);
    if (e != hipSuccess) {
        iwp_tensors_destroy(t);
        return hip_fail(e, "iwp_tensors_create");
    }
    *tensors_out = t;
    return IWP_OK;
}

void iwp_tensors_destroy(iwp_tensors* tensors) {
    if (!tensors) return;
    if (tensors->chunks) (void)hipFree(tensors->chunks);
    delete tensors;
}

size_t iwp_tensors_workspace_bytes(const iwp_tensors* tensors, uint32_t W) {
    if (!tensors || W < 1 || W > IWP_MAX_WORKERS) return 0;
    return ((size_t)W * blocks_of(tensors->n_chunks, W) * sizeof(double) + 255) & ~size_t(255);
}

int iwp_clip(const iwp_tensors* tensors, const float* const* g, float* const* out, uint32_t W, double scale, double max_norm, float* norm,
             void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (!tensors || !g || W < 1 || W > IWP_MAX_WORKERS || !norm) return IWP_EINVAL;
    if (!std::isfinite(scale) || !(max_norm >= 0.0)) return IWP_EINVAL;
    if (!aligned(norm, 4) || !aligned(workspace, 256)) return IWP_EALIGN;
    bool writes = false;
    ClipCall c{tensors->chunks, tensors->n_chunks, blocks_of(tensors->n_chunks, W), scale, max_norm, norm, static_cast<double*>(workspace), {}, {}};
    for (uint32_t p = 0; p < W; ++p) {
        c.g[p] = g[p];
        c.out[p] = out && g[p] ? out[p] : nullptr;
        writes |= c.out[p] != nullptr;
        if (!aligned(c.g[p], 4) || !aligned(c.out[p], 4)) return IWP_EALIGN;
    }
    // what a worker writes is nobody else's, and not a shifted part of its own gradient
    const uint64_t length = (tensors->end - tensors->begin) * sizeof(float);
    auto apart = [&](const float* a, const float* b) {
        const uint64_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
        return x >= y ? x - y >= length : y - x >= length;
    };
    for (uint32_t p = 0; p < W; ++p)
        for (uint32_t q = 0; c.out[p] && q < W; ++q) {
            if (q != p && c.out[q] && !apart(c.out[p], c.out[q])) return IWP_EINVAL;
            if (c.g[q] && !(q == p && c.out[p] == c.g[p]) && !apart(c.out[p], c.g[q])) return IWP_EINVAL;
        }
    if (!workspace || workspace_bytes < iwp_tensors_workspace_bytes(tensors, W)) return IWP_EWORKSPACE;
    const hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (c.n_chunks <= ONE_CHUNKS) {
        IWP_LAUNCH_BLOCK("k_clip_one", k_clip_one, W, 1024, s, c);
        return IWP_OK;
    }
    const uint32_t together = writes ? at_a_time(c.n_chunks, W) : W;
    if (!writes) c.blocks = std::min(c.blocks, std::max(1u, GRID / W));
    const uint32_t blocks = writes ? c.blocks : 1;
    const bool past_cache = W * worker_bytes(c.n_chunks) > CACHE_BYTES;
    for (uint32_t first = 0; first < W; first += together) {
        const uint32_t workers = std::min(together, W - first);
        IWP_LAUNCH_BLOCK("k_clip_norm", k_clip_norm, workers * c.blocks, 256, s, c, first);
        auto apply = past_cache ? k_clip_apply<true> : k_clip_apply<false>;
        IWP_LAUNCH_BLOCK("k_clip_apply", apply, workers * blocks, 256, s, c, first, blocks);
    }
    return IWP_OK;
}

}  // extern "C"
