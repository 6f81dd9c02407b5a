// Penalties, biases and grammar masks on logits, with each row's first maximum.
//
//   constrain_kernel  one workgroup per (tree node, 8192 tokens of the vocabulary).  The node's path is walked in LDS and its tokens are
//                     counted into a table of the chunk; then the chunk streams through once, four logits to a thread and step, each
//                     with its confirmed count, path count, bias and mask bit.  The arithmetic is fp32, one rounding per step as
//                     the definition has it (no fused multiply-add), so that equal inputs give equal ties.
//   best_kernel       the chunks' maxima of a row, first maximum.
// Counts and biases of a sequence are read by all of its nodes and stay in L2.  129 rows of
// 128256 bf16 logits with everything on: 25.3 us with both kernels (a copy of their size takes 18), 784 rows of 32003 fp32 logits read for
// their maxima only 31.9.  Both are bound by vector instructions: 42 to 44 per logit, with which the SIMDs are busy all the time
// (counted).  Many resident wavefronts with few registers serve best: four rows to a workgroup that share counts and biases, or
// all of a thread's loads up front, or penalties for listed tokens only, measured 41 to 60 us.  The logits are stored past the caches: with
// plain stores 35 us instead of 25, though a reader that follows at once (an argmax over them) then ends 3 us earlier (50.7 and 53.7 us
// for both).
#include "ygg_internal.h"
#include "ygg_device.h"

#include <algorithm>
#include <type_traits>

namespace ygg {
namespace {

constexpr int kChunk = 8192;

// A row's (or a chunk's) maximum: larger values have larger keys, the two zeros the same one, a NaN the largest.
struct Best {
    uint32_t key;
    int32_t idx;
};
__device__ __forceinline__ uint32_t rank_of(float v) { return v != v ? 0xffffffffu : key_of(v + 0.f); }   // (-0 + 0 = 0)
// The largest key in the wavefront, and the lowest index that has it.
__device__ __forceinline__ Best first_of_wave(uint32_t key, int32_t idx) {
    const uint32_t top = wave_max_u32(key);
    return {top, (int32_t)wave_min_u32(key == top ? (uint32_t)idx : 0x7fffffffu)};
}

// Rows start at any element, so vectors are only as aligned as their elements.
struct __attribute__((packed, aligned(4))) F4 { float x[4]; };
struct __attribute__((packed, aligned(4))) I4 { int32_t x[4]; };
struct __attribute__((packed, aligned(2))) H4 { uint16_t x[4]; };
typedef float Out4 __attribute__((ext_vector_type(4), aligned(4)));

template <typename T>
__device__ __forceinline__ float logit_of(T v) {
    if constexpr (sizeof(T) == 4) return v;
    else return __uint_as_float((uint32_t)v << 16);
}

// x / d, correctly rounded, for many x > 0: Markstein's method from the correctly rounded reciprocal r of d -- a quotient within one unit
// of the last place, corrected by its exact remainder (twice: the first correction brings the quotient that near).  It holds for d from
// 2^-32 to 2^32 and quotients from 2^-64 to 2^120, where no remainder (a multiple of 2^(-64-23-32-23) = 2^-142) leaves fp32's range; others
// want the division itself.
struct Divisor {
    float d, r;
    uint32_t span;      // of the bits of such quotients; 0: no quotient by this d
    __device__ __forceinline__ explicit Divisor(float x) : d(x), r(1.f / x), span(x >= 0x1p-32f && x <= 0x1p32f ? (uint32_t)(120 + 64) << 23 : 0) {}
    __device__ __forceinline__ float of(float x) const {
        float q = x * r;
        q = fmaf(fmaf(-q, d, x), r, q);
        return fmaf(fmaf(-q, d, x), r, q);
    }
    __device__ __forceinline__ bool fails(float q) const { return __float_as_uint(q) - ((127u - 64) << 23) >= span; }
};

template <typename T>
__global__ __launch_bounds__(256) void constrain_kernel(ConstrainArgs a) {
    extern __shared__ int32_t nodes_s[];                // parents, tokens
    int32_t *const parent_s = nodes_s, *const token_s = nodes_s + a.N;
    __shared__ __align__(16) uint16_t times_s[kChunk];   // occurrences on the path, by token of the chunk
    __shared__ Best best_s[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t row = blockIdx.x;   // b * N + i
    const int b = (int)(row / a.N), i = (int)(row - (int64_t)b * a.N);
    const int c0 = blockIdx.y * kChunk, c1 = min(a.V, c0 + kChunk);

    for (int n = tid; n <= i; n += 256) {
        parent_s[n] = a.parent_idx[(int64_t)b * a.N + n];
        token_s[n] = a.token_ids[(int64_t)b * a.N + n];
    }
    for (int n = tid; n < kChunk / 8; n += 256) reinterpret_cast<uint4*>(times_s)[n] = make_uint4(0, 0, 0, 0);
    const float repetition = a.repetition ? a.repetition[b] : 1.f;
    const float presence = a.presence ? a.presence[b] : 0.f, frequency = a.frequency ? a.frequency[b] : 0.f;
    const uint32_t* mask = nullptr;
    if (a.masks) {
        const int m = a.mask_index[row];
        if (m >= 0) mask = a.masks + (int64_t)min(m, a.n_masks - 1) * ((a.V + 31) / 32);
    }
    __syncthreads();
    if (tid == 0)
        for (int n = i;;) {   // a parent that is no earlier node ends the walk
            const int t = token_s[n];
            if (t >= c0 && t < c1) ++times_s[t - c0];
            const int p = parent_s[n];
            if (p < 0 || p >= n) break;
            n = p;
        }
    __syncthreads();

    const T* x = static_cast<const T*>(a.logits) + row * a.row_stride;
    const int32_t* counts = a.counts ? a.counts + (int64_t)b * a.V : nullptr;
    const float* bias = a.bias ? a.bias + (a.bias_shared ? 0 : (int64_t)b * a.V) : nullptr;
    float* out = a.out ? a.out + row * a.V : nullptr;
    float bv = -INFINITY;
    int bi = c0 + 4 * tid < c1 ? c0 + 4 * tid : 0x7fffffff;
    auto consider = [&](float y, int j) {   // the first maximum, or the first NaN
        if (!(y <= bv) && bv == bv) { bv = y; bi = j; }
    };
    const Divisor over(repetition);
    bool again = false;    // a quotient was none: these logits once more, with divisions
    auto constrained = [&](auto divide, float v, int32_t confirmed, uint32_t times, float add, bool allowed) {
#pragma clang fp contract(off)
        const uint32_t c = ((uint32_t)confirmed & 0x7fffffffu) + times;
        float q;
        if constexpr (divide) q = v / repetition;
        else {
            q = over.of(v);
            again |= v > 0.f && over.fails(q);
        }
        if (confirmed != 0 || times) v = v > 0.f ? q : v * repetition;
        v = v - frequency * (float)c;
        v = v - (c ? presence : 0.f);
        if (bias) v = v + add;
        return allowed ? v : -INFINITY;
    };
    typedef std::integral_constant<bool, false> Quotients;
    typedef std::integral_constant<bool, true> Divisions;
    for (int j = c0 + 4 * tid; j < c1; j += 1024) {
        if (j + 4 <= c1) {
            float v[4];
            if constexpr (sizeof(T) == 4) {
                const F4 q = *reinterpret_cast<const F4*>(x + j);
                for (int e = 0; e < 4; ++e) v[e] = q.x[e];
            } else {
                const H4 q = *reinterpret_cast<const H4*>(x + j);
                for (int e = 0; e < 4; ++e) v[e] = logit_of(q.x[e]);
            }
            I4 n = {};
            F4 add = {};
            if (counts) n = *reinterpret_cast<const I4*>(counts + j);
            if (bias) add = *reinterpret_cast<const F4*>(bias + j);
            const uint32_t bits = mask ? mask[j >> 5] >> (j & 31) : 0xfu;
            const uint2 times = *reinterpret_cast<const uint2*>(times_s + (j - c0));
            Out4 y;
            auto all = [&](auto divide) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t t = ((e < 2 ? times.x : times.y) >> (16 * (e & 1))) & 0xffffu;
                    y[e] = constrained(divide, v[e], n.x[e], t, add.x[e], (bits >> e) & 1u);
                }
            };
            again = false;
            all(Quotients{});
            if (again) all(Divisions{});
#pragma unroll
            for (int e = 0; e < 4; ++e) consider(y[e], j + e);
            if (out) __builtin_nontemporal_store(y, reinterpret_cast<Out4*>(out + j));
        } else {
            for (int e = j; e < c1; ++e) {
                const float y = constrained(Divisions{}, logit_of(x[e]), counts ? counts[e] : 0, times_s[e - c0], bias ? bias[e] : 0.f,
                                            !mask || ((mask[e >> 5] >> (e & 31)) & 1u));
                consider(y, e);
                if (out) out[e] = y;
            }
        }
    }
    if (!a.best) return;
    const Best mine = first_of_wave(rank_of(bv), bi);
    if (lane == 0) best_s[wave] = mine;
    __syncthreads();
    if (tid == 0) {
        Best best = mine;
#pragma unroll
        for (int w = 1; w < 4; ++w)
            if (best_s[w].key > best.key || (best_s[w].key == best.key && best_s[w].idx < best.idx)) best = best_s[w];
        if (gridDim.y == 1) a.best[row] = best.idx;
        else static_cast<Best*>(a.part)[row * gridDim.y + blockIdx.y] = best;
    }
}

__global__ __launch_bounds__(256) void best_kernel(ConstrainArgs a, int64_t rows, int chunks) {
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (row >= rows) return;
    const Best* p = static_cast<const Best*>(a.part) + row * chunks;
    Best best = {0, 0x7fffffff};
    for (int c = lane; c < chunks; c += 64)
        if (p[c].key > best.key) best = p[c];   // (a lane's chunks come in order)
    best = first_of_wave(best.key, best.idx);
    if (lane == 0) a.best[row] = best.idx;
}

__global__ __launch_bounds__(256) void count_kernel(CountArgs a) {
    const int b = blockIdx.y;
    const int n = min(a.n_new[b], a.max_new);
    for (int64_t k = blockIdx.x * 256 + threadIdx.x; k < n; k += gridDim.x * 256) {
        const int64_t r = a.rows ? (int64_t)a.rows[(int64_t)b * a.max_new + k] : a.first + k;
        if (r < 0 || r >= a.n_tokens) continue;
        const int t = a.tokens[(int64_t)b * a.n_tokens + r];
        if (t < 0 || t >= a.V) continue;
        int32_t* c = a.counts + (int64_t)b * a.V + t;
        if (a.prompt) atomicOr(c, (int32_t)0x80000000);
        else atomicAdd(c, 1);
    }
}

}  // namespace

size_t constrain_scratch_bytes(const ygg_shape& s) {
    const int64_t rows = (int64_t)s.batch * s.n_nodes, chunks = ((int64_t)s.vocab + kChunk - 1) / kChunk;
    return ((size_t)(rows * chunks) * sizeof(Best) + 255) / 256 * 256;
}

hipError_t launch_constrain(const ConstrainArgs& a, bool f32, hipStream_t st) {
    const int64_t rows = (int64_t)a.B * a.N;
    const int chunks = (a.V + kChunk - 1) / kChunk;
    const dim3 grid((unsigned)rows, (unsigned)chunks);
    if (f32) hipLaunchKernelGGL((constrain_kernel<float>), grid, dim3(256), 2 * a.N * sizeof(int32_t), st, a);
    else hipLaunchKernelGGL((constrain_kernel<uint16_t>), grid, dim3(256), 2 * a.N * sizeof(int32_t), st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.best || chunks == 1) return e;
    hipLaunchKernelGGL(best_kernel, dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, st, a, rows, chunks);
    return hipGetLastError();
}

hipError_t launch_count(const CountArgs& a, hipStream_t st) {
    const unsigned groups = (unsigned)std::clamp(((int64_t)a.max_new + 255) / 256, (int64_t)1, (int64_t)64);
    hipLaunchKernelGGL(count_kernel, dim3(groups, (unsigned)a.B), dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace ygg
