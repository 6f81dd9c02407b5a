// Appending tokens to the 4-bit block cache (include/ygg.h has the format).
//
// One workgroup per (layer, sequence, kv head, touched block), as for the 8-bit cache.  A thread takes eight dimensions of a token of K
// (four threads meet in their lanes for the 32 values of a scale) and eight dimensions of four tokens of V (sixteen lanes' worth of
// tokens meet there and, at head_dim 128, the two wavefronts of a half of the block through LDS).  Scales are powers of two that the
// conversion to E2M1 takes along, so a value costs half an instruction; codes and scales gather in LDS in the order in which they are stored.
// Bound by the stream of rows: 8191 tokens of a prompt, 4 layers of 8 kv heads of 128, 37.7 us, 4.5 TB/s; the accepted tokens of 16
// requests, 32 layers, 12.7 us.
#include "block_cache.h"

namespace ygg {
namespace {

using namespace block_cache;

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(8))) uint16_t u16x8;

// Exponent + 127 of the least 2^e >= 2^-100 with amax <= 7 * 2^e, from the bits of a bf16: a significand above 1.75 (0x60 of 0x80) carries.
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax) { return (uint32_t)max((int)((amax + 0x1f) >> 7) - 2, 27); }
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }
__device__ __forceinline__ uint32_t max_u32(uint32_t x, uint32_t y) { return x > y ? x : y; }
// The two bf16 of `pair` as codes in byte AT of w.
template <int AT>
__device__ __forceinline__ uint32_t encode2(uint32_t w, uint32_t pair, float scale) {
    return (uint32_t)__builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, pair), scale, AT);
}

template <int DH>
__global__ __launch_bounds__(256) void block4_append_kernel(AppendArgs a) {
    constexpr int OCT = DH / 8;                  // pieces of eight dimensions of a row
    constexpr int PT = kT * OCT / 256;           // K: pieces to a thread
    constexpr int CODES = kT * DH / 2;           // bytes of a block's K (or V)
    constexpr int SCALES = 2 * DH;
    constexpr int PER_HALF = DH == 128 ? 2 : 1;  // wavefronts that share 32 tokens of V
    __shared__ __align__(16) unsigned char code_s[2][CODES];
    __shared__ __align__(16) unsigned char scale_s[2][SCALES];
    __shared__ __align__(16) uint16_t top_s[4][DH];
    const int tid = threadIdx.x, wave = tid >> 6;
    const Touched x(a, DH);

    if (x.complete) {
        u32x4 k[PT], v[4];
#pragma unroll
        for (int u = 0; u < PT; ++u) {
            const int p = tid + 256 * u;
            k[u] = fetch(x.k_row(x.t0 + p / OCT), p % OCT * 8);
        }
        const int oct = tid % OCT, quad = tid / OCT;     // (head_dim 64: the second half of the threads has none)
#pragma unroll
        for (int t = 0; t < 4; ++t) v[t] = quad < 16 ? fetch(x.v_row(x.t0 + 4 * quad + t), 8 * oct) : u32x4{};

        // K: the 32 dimensions of a scale are four neighbouring threads'
#pragma unroll
        for (int u = 0; u < PT; ++u) {
            const int p = tid + 256 * u, t = p / OCT, o = p % OCT;
            const u16x2 m = magnitude8(k[u], u16x2{});
            uint32_t top = max_u32(m[0], m[1]);
            top = max_u32(top, row_xor<1>(top));
            top = max_u32(top, row_xor<2>(top));
            const uint32_t byte = scale_byte(top);
            const float scale = scale_of(byte);
            uint32_t w = encode2<0>(k[u][0], k[u][0], scale);      // (every byte is overwritten)
            w = encode2<1>(w, k[u][1], scale);
            w = encode2<2>(w, k[u][2], scale);
            w = encode2<3>(w, k[u][3], scale);
            const int chunk = t / 32 * (DH / 64) + o / 8, to = 32 * (o / 4 % 2) + t % 32;
            // in LDS a chunk's tokens lie permuted by the quarter of the row, or the quarters would meet on the same banks
            *reinterpret_cast<uint32_t*>(code_s[0] + 1024 * chunk + 16 * (to ^ (o / 4 << 2)) + 4 * (o % 4)) = w;
            if (o % 4 == 0) scale_s[0][to * (DH / 32) + chunk] = (unsigned char)byte;
        }
        // V: per dimension over 32 tokens: a thread's four, the lanes of the same eight dimensions, then the other wavefront
        u16x2 top[4] = {};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
#pragma unroll
            for (int t = 0; t < 4; ++t) top[e] = __builtin_elementwise_max(top[e], __builtin_bit_cast(u16x2, v[t][e] & 0x7fff7fffu));
            auto meet = [&](uint32_t other) { top[e] = __builtin_elementwise_max(top[e], __builtin_bit_cast(u16x2, other)); };
            if constexpr (OCT == 8) meet(lane_xor<8>(__builtin_bit_cast(uint32_t, top[e])));
            meet(lane_xor<16>(__builtin_bit_cast(uint32_t, top[e])));
            meet(lane_xor<32>(__builtin_bit_cast(uint32_t, top[e])));
        }
        if ((tid & 63) < OCT) *reinterpret_cast<u32x4*>(&top_s[wave][8 * oct]) = __builtin_bit_cast(u32x4, top);
        __syncthreads();
        if (quad < 16) {
            const int half = quad / 8;
            u16x8 both = {};
#pragma unroll
            for (int i = 0; i < PER_HALF; ++i) both = __builtin_elementwise_max(both, *reinterpret_cast<const u16x8*>(&top_s[PER_HALF * half + i][8 * oct]));
            // four codes of dimension 8 oct + e: chunk oct / 4, lane 32 half + 8 (oct % 4) + e, half a word at 4 (quad % 2) + quad % 8 / 2;
            // in LDS the lanes of eight dimensions lie permuted by oct, or all of a wavefront's octets would meet one bank
            const int lane0 = 32 * half + 8 * (oct % 4);
            unsigned char* const to = code_s[1] + 1024 * (oct / 4) + 16 * lane0 + 8 * (quad % 2) + 2 * (quad % 8 / 2);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t byte = scale_byte(both[e]);
                const float scale = scale_of(byte);
                constexpr uint32_t kLow = 0x05040100, kHigh = 0x07060302;
                const uint32_t pick = e % 2 ? kHigh : kLow;
                uint32_t w = encode2<0>(0, __builtin_amdgcn_perm(v[1][e / 2], v[0][e / 2], pick), scale);
                w = encode2<1>(w, __builtin_amdgcn_perm(v[3][e / 2], v[2][e / 2], pick), scale);
                *reinterpret_cast<uint16_t*>(to + 16 * (e ^ (oct & 7))) = (uint16_t)w;
                if (quad % 8 == 0) scale_s[1][(lane0 + e) * (DH / 32) + oct / 4] = (unsigned char)byte;
            }
        }
        __syncthreads();
        unsigned char* const kc = static_cast<unsigned char*>(a.k_codes) + x.at * CODES;
        unsigned char* const vc = static_cast<unsigned char*>(a.v_codes) + x.at * CODES;
        for (int p = tid; p < CODES / 16; p += 256) {
            const int chunk = p / 64, from = p % 64;
            const int quarter = 2 * (chunk % (DH / 64)) + from / 32, octet = 4 * chunk + from % 32 / 8;
            __builtin_nontemporal_store(*reinterpret_cast<const u32x4*>(code_s[0] + 1024 * chunk + 16 * (from ^ (quarter << 2))), reinterpret_cast<u32x4*>(kc + 16 * p));
            __builtin_nontemporal_store(*reinterpret_cast<const u32x4*>(code_s[1] + 1024 * chunk + 16 * (from ^ (octet & 7))), reinterpret_cast<u32x4*>(vc + 16 * p));
        }
        if (tid < 2 * SCALES / 16) {
            const int is_v = tid / (SCALES / 16), p = tid % (SCALES / 16);
            unsigned char* const to = static_cast<unsigned char*>(is_v ? a.v_scale : a.k_scale) + x.at * SCALES;
            *reinterpret_cast<u32x4*>(to + 16 * p) = *reinterpret_cast<const u32x4*>(scale_s[is_v] + 16 * p);
        }
    }
    x.keep_open_rows(a, tid);
}

}  // namespace

hipError_t launch_block4_append(const AppendArgs& a, int head_dim, hipStream_t st) {
    const dim3 grid((unsigned)((int64_t)a.n_layers * a.B * a.Hkv * a.blocks));
    if (head_dim == 128) hipLaunchKernelGGL((block4_append_kernel<128>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((block4_append_kernel<64>), grid, dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace ygg
