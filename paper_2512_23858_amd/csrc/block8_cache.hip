// Appending tokens to the 8-bit block cache (include/ygg.h has the format).
//
// One workgroup per (layer, sequence, kv head, touched block).  A block that the new tokens complete is read once, old rows from the
// tail and new ones from the caller's tensor, its largest magnitudes are reduced over the workgroup, and its codes are written in the
// order in which the attention's matrix instructions take them.  K: a thread has 16 dimensions of one token, which are 16 consecutive
// bytes there, so codes go from registers to memory.  V: 16 tokens of one dimension are, so a thread has eight dimensions of four
// tokens, transposes them in registers to words of four tokens, and the words meet in LDS (gathered there byte by byte they took half
// as many instructions again as all the rest).  The workgroup of the first touched block also copies the rows that stay open to the
// tail, after it has read that block's old rows: they may lie in the same half of it.  Bound by the stream of rows: 8191 tokens of four
// layers and 8 kv heads of 128 45.4 us, 4.4 TB/s of rows and codes; the accepted tokens of 16 requests in 32 layers 14 to 16 us, most of its
// bytes being the rows of completed blocks.
#include "ygg_internal.h"
#include "ygg_device.h"

namespace ygg {
namespace {

constexpr int kT = YGG_KV_BLOCK;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;

__device__ __forceinline__ float bf16_lo(uint32_t d) { return __uint_as_float(d << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t d) { return __uint_as_float(d & 0xffff0000u); }

// E4M3 codes of the four values of two words, times inv.
__device__ __forceinline__ uint32_t encode4(uint32_t p, uint32_t q, float inv) {
    const int w = __builtin_amdgcn_cvt_pk_fp8_f32(bf16_lo(p) * inv, bf16_hi(p) * inv, (int)p, false);   // (both halves of p are overwritten)
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(bf16_lo(q) * inv, bf16_hi(q) * inv, w, true);
}
__device__ __forceinline__ u32x4 encode16(const u32x4 lo, const u32x4 hi, float inv) {
    return u32x4{encode4(lo[0], lo[1], inv), encode4(lo[2], lo[3], inv), encode4(hi[0], hi[1], inv), encode4(hi[2], hi[3], inv)};
}
// Byte k of the four words in word k: words of four dimensions of a token <-> words of four tokens of a dimension.
__device__ __forceinline__ void transpose4(uint32_t (&w)[4]) {
    const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400), b = __builtin_amdgcn_perm(w[1], w[0], 0x07030602);
    const uint32_t c = __builtin_amdgcn_perm(w[3], w[2], 0x05010400), d = __builtin_amdgcn_perm(w[3], w[2], 0x07030602);
    w[0] = __builtin_amdgcn_perm(c, a, 0x05040100);
    w[1] = __builtin_amdgcn_perm(c, a, 0x07060302);
    w[2] = __builtin_amdgcn_perm(d, b, 0x05040100);
    w[3] = __builtin_amdgcn_perm(d, b, 0x07060302);
}
// The largest bits of the magnitudes of eight values in either half of a word (magnitudes are in the order of their bits).
__device__ __forceinline__ u16x2 magnitude8(const u32x4 v, u16x2 m) {
#pragma unroll
    for (int e = 0; e < 4; ++e) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, v[e] & 0x7fff7fffu));
    return m;
}
__device__ __forceinline__ float largest(u16x2 m) { return __uint_as_float((uint32_t)max(m[0], m[1]) << 16); }
// at least 2^-100: the attention splits a scale into its exponent and its significand
__device__ __forceinline__ float scale_of(float amax) { return amax > 0.f ? fmaxf(amax / 448.f, 7.888609052210118e-31f) : 1.f; }

template <int DH>
__global__ __launch_bounds__(256) void block8_append_kernel(AppendArgs a) {
    constexpr int P = kT * DH / 16;       // pieces of 16 elements in a block
    constexpr int PT = P / 256;           // per thread
    constexpr int PR = DH / 16;           // per row
    constexpr int OCT = DH / 8;   // V: eight dimensions of four tokens to a thread
    __shared__ __align__(16) unsigned char v_s[kT * DH];
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
        auto row_at = [&](int64_t token, const uint16_t* tail, const uint16_t* fresh_rows) -> const uint16_t* {   // or null: zeros
            if (token < old) return tail + token % (2 * kT) * row;
            const int64_t r = new_row(token);
            return r >= 0 ? fresh_rows + r * row : nullptr;
        };
        auto fetch = [](const uint16_t* p, int d) {
            u32x4 x = {};
            if (p) x = *reinterpret_cast<const u32x4*>(p + d);
            return x;
        };
        u32x4 k[PT][2], v[4];
#pragma unroll
        for (int u = 0; u < PT; ++u) {
            const int p = tid + 256 * u, t = p / PR, d = p % PR * 16;
            const uint16_t* const src = row_at(t0 + t, k_tail, k_new);
            k[u][0] = fetch(src, d);
            k[u][1] = fetch(src, d + 8);
        }
        const int oct = tid % OCT, quad = tid / OCT;     // (head_dim 64: the second half of the threads has none)
#pragma unroll
        for (int t = 0; t < 4; ++t) v[t] = quad < 16 ? fetch(row_at(t0 + 4 * quad + t, v_tail, v_new), 8 * oct) : u32x4{};
        u16x2 km = {}, vm = {};
#pragma unroll
        for (int u = 0; u < PT; ++u) km = magnitude8(k[u][1], magnitude8(k[u][0], km));
#pragma unroll
        for (int t = 0; t < 4; ++t) vm = magnitude8(v[t], vm);
        auto larger = [](float x, float y) { return fmaxf(x, y); };
        const float kw = group_reduce(largest(km), 64, larger), vw = group_reduce(largest(vm), 64, larger);
        if (lane == 0) { amax_s[0][wave] = kw; amax_s[1][wave] = vw; }
        __syncthreads();
        const float ks = scale_of(fmaxf(fmaxf(amax_s[0][0], amax_s[0][1]), fmaxf(amax_s[0][2], amax_s[0][3])));
        const float vs = scale_of(fmaxf(fmaxf(amax_s[1][0], amax_s[1][1]), fmaxf(amax_s[1][2], amax_s[1][3])));
        const float ki = 1.f / ks, vi = 1.f / vs;
        const int64_t at = (lb * a.Hkv + g) * a.nblk + block;
        unsigned char* const kc = static_cast<unsigned char*>(a.k_codes) + at * kT * DH;
        unsigned char* const vc = static_cast<unsigned char*>(a.v_codes) + at * kT * DH;
        if (tid == 0) { a.k_scale[at] = ks; a.v_scale[at] = vs; }
        // Codes are stored past the caches (54.0 -> 50.8 us for 8191 tokens of four layers; streaming loads of the rows cost 3).
#pragma unroll
        for (int u = 0; u < PT; ++u) {
            const int p = tid + 256 * u, t = p / PR, d = p % PR * 16;
            const int chunk = 2 * ((t / 32) * (DH / 64) + d / 64) + d / 16 % 2, to = 32 * (d / 32 % 2) + t % 32;
            __builtin_nontemporal_store(encode16(k[u][0], k[u][1], ki), reinterpret_cast<u32x4*>(kc + 1024 * chunk + 16 * to));
        }
        if (quad < 16) {
            // word of tokens 4 quad .. + 3 and dimension 8 oct + e: chunk 2 (d / 32) + quad / 8, lane 32 (quad % 2) + d % 32, word quad % 8 / 2;
            // in LDS the lanes of eight dimensions lie permuted by oct, or all of a wavefront's octets would meet one bank
            unsigned char* const to = v_s + 1024 * (2 * (oct / 4) + quad / 8) + 16 * (32 * (quad % 2) + 8 * (oct % 4)) + 4 * (quad % 8 / 2);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t words[4];
#pragma unroll
                for (int t = 0; t < 4; ++t) words[t] = encode4(v[t][2 * h], v[t][2 * h + 1], vi);
                transpose4(words);
#pragma unroll
                for (int e = 0; e < 4; ++e) *reinterpret_cast<uint32_t*>(to + 16 * ((4 * h + e) ^ (oct & 7))) = words[e];
            }
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < PT; ++u) {
            const int p = tid + 256 * u, chunk = p / 64, from = p % 64, octet = 4 * (chunk / 2) + from % 32 / 8;
            const u32x4 codes = *reinterpret_cast<const u32x4*>(v_s + 1024 * chunk + 16 * (from ^ (octet & 7)));
            __builtin_nontemporal_store(codes, reinterpret_cast<u32x4*>(vc + 16 * p));
        }
    }
    if (j > 0) return;
    // rows that stay open (those that complete a block are in its codes, and nothing reads them from here: the header says how far back a
    // length may be taken)
    const int64_t open = max(end / kT * kT, old);
    for (int64_t p = tid; p < (end - open) * (DH / 8); p += 256) {
        const int64_t token = open + p / (DH / 8), r = new_row(token);
        const int64_t d = p % (DH / 8) * 8;
        u32x4 k = {}, v = {};
        if (r >= 0) {
            k = *reinterpret_cast<const u32x4*>(k_new + r * row + d);
            v = *reinterpret_cast<const u32x4*>(v_new + r * row + d);
        }
        *reinterpret_cast<u32x4*>(k_tail + token % (2 * kT) * row + d) = k;
        *reinterpret_cast<u32x4*>(v_tail + token % (2 * kT) * row + d) = v;
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
