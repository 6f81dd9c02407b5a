// Appending tokens to the 8-bit block cache (include/ygg.h has the format).
//
// One workgroup per (layer, sequence, kv head, touched block).  A block that the new tokens complete is read once, old rows from the
// tail and new ones from the caller's tensor, its largest magnitudes are reduced over the workgroup, and its codes are written in the
// order in which the attention's matrix instructions take them.  K: a thread's 16 dimensions of one token are 16 consecutive bytes
// there, so codes go from registers to memory.  V: 16 tokens of one dimension are, so codes pass through LDS.  The workgroup of the
// first touched block also copies the rows that stay open to the tail, after it has read that block's old rows: they may lie in the
// same half of it.  Bound by the stream of rows.
#include "ygg_internal.h"
#include "ygg_device.h"

namespace ygg {
namespace {

constexpr int kT = YGG_KV_BLOCK;

__device__ __forceinline__ float bf16_lo(uint32_t d) { return __uint_as_float(d << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t d) { return __uint_as_float(d & 0xffff0000u); }

// E4M3 codes of four values, nearest to x / scale: the product with the reciprocal, corrected once by its remainder.
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d, float scale, float inv) {
    auto quotient = [&](float x) {
        const float q = x * inv;
        return fmaf(fmaf(-q, scale, x), inv, q);
    };
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(quotient(a), quotient(b), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(quotient(c), quotient(d), w, true);
}
__device__ __forceinline__ uint4 encode16(const uint4 lo, const uint4 hi, float scale, float inv) {
    auto two = [&](uint32_t p, uint32_t q) { return encode4(bf16_lo(p), bf16_hi(p), bf16_lo(q), bf16_hi(q), scale, inv); };
    return make_uint4(two(lo.x, lo.y), two(lo.z, lo.w), two(hi.x, hi.y), two(hi.z, hi.w));
}
__device__ __forceinline__ float magnitude8(const uint4 v, float m) {
    const uint32_t d[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) m = fmaxf(m, fmaxf(fabsf(bf16_lo(d[e])), fabsf(bf16_hi(d[e]))));
    return m;
}
// at least 2^-100: the attention splits a scale into its exponent and its significand
__device__ __forceinline__ float scale_of(float amax) { return amax > 0.f ? fmaxf(amax / 448.f, 7.888609052210118e-31f) : 1.f; }

template <int DH>
__global__ __launch_bounds__(256) void block8_append_kernel(AppendArgs a) {
    constexpr int P = kT * DH / 16;       // pieces of 16 elements in a block
    constexpr int PT = P / 256;           // per thread
    constexpr int PR = DH / 16;           // per row
    constexpr int VROW = DH + 16;         // bytes of a row of V's codes in LDS
    __shared__ __align__(16) unsigned char v_s[kT * VROW];
    __shared__ float amax_s[2][4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int64_t w = blockIdx.x;
    const int j = (int)(w % a.blocks); w /= a.blocks;
    const int g = (int)(w % a.Hkv); w /= a.Hkv;
    const int b = (int)(w % a.B);
    const int64_t lb = w;                 // layer * B + b

    const int64_t len = a.seq_lens[b];
    const int64_t end = len < 0 ? 0 : (len > a.cap ? a.cap : len);
    const int64_t want = a.n_new[b];
    int64_t fresh = want < 0 ? 0 : (want > a.max_new ? a.max_new : want);
    if (fresh > end) fresh = end;
    const int64_t old = end - fresh;
    const int64_t block = old / kT + j;
    const int64_t t0 = block * kT;        // the block's first token
    const bool complete = t0 + kT <= end && fresh > 0;

    const int64_t row = (int64_t)a.Hkv * DH;
    const uint16_t* const k_new = static_cast<const uint16_t*>(a.k_new) + lb * a.n_rows * row + (int64_t)g * DH;
    const uint16_t* const v_new = static_cast<const uint16_t*>(a.v_new) + lb * a.n_rows * row + (int64_t)g * DH;
    uint16_t* const k_tail = static_cast<uint16_t*>(a.k_tail) + lb * 2 * kT * row + (int64_t)g * DH;
    uint16_t* const v_tail = static_cast<uint16_t*>(a.v_tail) + lb * 2 * kT * row + (int64_t)g * DH;
    auto new_row = [&](int64_t token) -> int64_t {   // row of the caller's tensor, or -1
        const int64_t k = token - old;
        const int64_t r = a.rows ? (int64_t)a.rows[(int64_t)b * a.max_new + k] : k;
        return r >= 0 && r < a.n_rows ? r : -1;
    };

    if (complete) {
        uint4 k[PT][2], v[PT][2];
#pragma unroll
        for (int u = 0; u < PT; ++u) {
            const int p = tid + 256 * u, t = p / PR, d = p % PR * 16;
            const int64_t token = t0 + t;
            const uint16_t *ks = nullptr, *vs = nullptr;
            if (token < old) {
                ks = k_tail + token % (2 * kT) * row;
                vs = v_tail + token % (2 * kT) * row;
            } else if (const int64_t r = new_row(token); r >= 0) {
                ks = k_new + r * row;
                vs = v_new + r * row;
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                k[u][h] = ks ? *reinterpret_cast<const uint4*>(ks + d + 8 * h) : make_uint4(0, 0, 0, 0);
                v[u][h] = vs ? *reinterpret_cast<const uint4*>(vs + d + 8 * h) : make_uint4(0, 0, 0, 0);
            }
        }
        float km = 0.f, vm = 0.f;
#pragma unroll
        for (int u = 0; u < PT; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                km = magnitude8(k[u][h], km);
                vm = magnitude8(v[u][h], vm);
            }
        auto larger = [](float x, float y) { return fmaxf(x, y); };
        km = group_reduce(km, 64, larger);
        vm = group_reduce(vm, 64, larger);
        if (lane == 0) { amax_s[0][wave] = km; amax_s[1][wave] = vm; }
        __syncthreads();
        const float ks = scale_of(fmaxf(fmaxf(amax_s[0][0], amax_s[0][1]), fmaxf(amax_s[0][2], amax_s[0][3])));
        const float vs = scale_of(fmaxf(fmaxf(amax_s[1][0], amax_s[1][1]), fmaxf(amax_s[1][2], amax_s[1][3])));
        const float ki = 1.f / ks, vi = 1.f / vs;
        const int64_t at = (lb * a.Hkv + g) * a.nblk + block;
        unsigned char* const kc = static_cast<unsigned char*>(a.k_codes) + at * kT * DH;
        unsigned char* const vc = static_cast<unsigned char*>(a.v_codes) + at * kT * DH;
        if (tid == 0) { a.k_scale[at] = ks; a.v_scale[at] = vs; }
#pragma unroll
        for (int u = 0; u < PT; ++u) {
            const int p = tid + 256 * u, t = p / PR, d = p % PR * 16;
            const int chunk = 2 * ((t / 32) * (DH / 64) + d / 64) + d / 16 % 2, to = 32 * (d / 32 % 2) + t % 32;
            *reinterpret_cast<uint4*>(kc + 1024 * chunk + 16 * to) = encode16(k[u][0], k[u][1], ks, ki);
            *reinterpret_cast<uint4*>(v_s + t * VROW + d) = encode16(v[u][0], v[u][1], vs, vi);
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < PT; ++u) {
            const int p = tid + 256 * u, chunk = p / 64, from = p % 64;
            const unsigned char* src = v_s + (32 * (chunk % 2) + 4 * (from / 32)) * VROW + 32 * (chunk / 2) + from % 32;
            uint32_t out[4];
#pragma unroll
            for (int e4 = 0; e4 < 4; ++e4) {
                out[e4] = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) out[e4] |= (uint32_t)src[(8 * e4 + e) * VROW] << (8 * e);
            }
            *reinterpret_cast<uint4*>(vc + 16 * p) = make_uint4(out[0], out[1], out[2], out[3]);
        }
    }
    if (j > 0) return;
    // rows that stay open
    const int64_t open = max(end / kT * kT, old);
    for (int64_t p = tid; p < (end - open) * (DH / 8); p += 256) {
        const int64_t token = open + p / (DH / 8), r = new_row(token);
        const int64_t d = p % (DH / 8) * 8;
        const uint4 zero = make_uint4(0, 0, 0, 0);
        *reinterpret_cast<uint4*>(k_tail + token % (2 * kT) * row + d) = r >= 0 ? *reinterpret_cast<const uint4*>(k_new + r * row + d) : zero;
        *reinterpret_cast<uint4*>(v_tail + token % (2 * kT) * row + d) = r >= 0 ? *reinterpret_cast<const uint4*>(v_new + r * row + d) : zero;
    }
}

}  // namespace

hipError_t launch_block8_append(const AppendArgs& a, int head_dim, hipStream_t st) {
    const dim3 grid((unsigned)((int64_t)a.n_layers * a.B * a.Hkv * a.blocks));
    if (head_dim == 128) hipLaunchKernelGGL((block8_append_kernel<128>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((block8_append_kernel<64>), grid, dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace ygg
