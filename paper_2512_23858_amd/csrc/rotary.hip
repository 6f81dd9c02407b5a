// Rotary positions of queries and keys (tree nodes: confirmed length + depth; or explicit positions).
//
// A wavefront takes one token, or a part of its heads where there are few tokens.  Its lanes first form the token's angles, one pair
// each: the turn p * f / 2 pi in fp64 (at position 10^6 an fp32 angle is off by 0.03 radians), its fraction of a whole turn, then
// sine and cosine of that in fp32.  Then a lane takes units of eight pairs -- two pieces of 16 bytes (fp32: 32) that lie half the
// rotated part apart, or next to each other where pairs are interleaved -- so that no value has to change lanes.  Bound by the stream
// of q and k; the unrotated part of a head passes through the same units.  2 x 8191 tokens of 40 heads of 128, bf16: 68.2 us, 4.9 TB/s, a
// copy's rate (past the caches it takes 81); 49 nodes for 16 requests of 72 heads 7.3 us; one token 2.2.
#include "ygg_internal.h"

#include <hip/hip_bf16.h>

#include <algorithm>

namespace ygg {
namespace {

constexpr int kTokens = 4;   // wavefronts, and so tokens, of a workgroup

struct Vec8 { float x[8]; };

template <typename T>
__device__ __forceinline__ Vec8 load8(const T* p) {
    Vec8 v;
    if constexpr (sizeof(T) == 4) {
        const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
        v.x[0] = a.x; v.x[1] = a.y; v.x[2] = a.z; v.x[3] = a.w; v.x[4] = b.x; v.x[5] = b.y; v.x[6] = b.z; v.x[7] = b.w;
    } else {
        const uint4 a = *reinterpret_cast<const uint4*>(p);
        const uint32_t d[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v.x[2 * e] = __uint_as_float(d[e] << 16);
            v.x[2 * e + 1] = __uint_as_float(d[e] & 0xffff0000u);
        }
    }
    return v;
}

template <typename T>
__device__ __forceinline__ void store8(T* p, const Vec8& v) {
    if constexpr (sizeof(T) == 4) {
        reinterpret_cast<float4*>(p)[0] = make_float4(v.x[0], v.x[1], v.x[2], v.x[3]);
        reinterpret_cast<float4*>(p)[1] = make_float4(v.x[4], v.x[5], v.x[6], v.x[7]);
    } else {
        __hip_bfloat16 h[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = __float2bfloat16(v.x[e]);   // round to nearest even
        *reinterpret_cast<uint4*>(p) = *reinterpret_cast<uint4*>(h);
    }
}

template <typename T, bool INTERLEAVED>
__global__ __launch_bounds__(kTokens * 64) void rotary_kernel(RotaryArgs a) {
    __shared__ int32_t parent_s[kMaxNodes];
    __shared__ float2 turn_s[kTokens][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int b = blockIdx.y;
    const int token = blockIdx.x * kTokens + wave;
    const int i = min(token, a.N - 1);

    int position;
    if (a.positions) {
        position = a.positions[(int64_t)b * a.N + i];
    } else {
        for (int j = tid; j < a.N; j += kTokens * 64) parent_s[j] = a.parent_idx[(int64_t)b * a.N + j];
        const int L = a.seq_lens[b];
        __syncthreads();
        position = L < 0 ? 0 : (L > a.max_seq_len ? a.max_seq_len : L);
        for (int n = i;;) {   // a parent that is no earlier node ends the walk
            const int p = parent_s[n];
            if (p < 0 || p >= n) break;
            n = p;
            ++position;
        }
    }
    const int pairs = a.rotary_dim / 2;
    if (lane < pairs) {
        const double turn = (double)position * (a.frequencies[lane] * 0.15915494309189533577);   // 1 / 2 pi
        float s, c;
        sincospif((float)(2.0 * (turn - rint(turn))), &s, &c);
        turn_s[wave][lane] = make_float2(c * a.scale, s * a.scale);
    }
    __syncthreads();
    if (token >= a.N) return;

    const int per_head = a.Dh / 16, rotated = a.rotary_dim / 16;
    const int64_t row = (int64_t)b * a.N + token;
    for (int u = blockIdx.z * 64 + lane; u < a.units; u += gridDim.z * 64) {
        const int head = u / per_head, k = u - head * per_head;
        const bool is_q = head < a.Hq;
        const T* src = is_q ? static_cast<const T*>(a.q) + row * a.q_stride + head * a.Dh
                            : static_cast<const T*>(a.k) + row * a.k_stride + (head - a.Hq) * a.Dh;
        T* dst = is_q ? static_cast<T*>(a.q_out) + (row * a.Hq + head) * a.Dh
                      : static_cast<T*>(a.k_out) + (row * a.Hkv + head - a.Hq) * a.Dh;
        const bool turned = k < rotated;
        const int first = !INTERLEAVED && turned ? 8 * k : 16 * k;
        const int second = !INTERLEAVED && turned ? 8 * k + pairs : 16 * k + 8;
        Vec8 x = load8(src + first), y = load8(src + second);
        if (turned) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float2 t = turn_s[wave][8 * k + e];
                if constexpr (INTERLEAVED) {
                    Vec8& v = e < 4 ? x : y;
                    const float p = v.x[2 * (e % 4)], q = v.x[2 * (e % 4) + 1];
                    v.x[2 * (e % 4)] = p * t.x - q * t.y;
                    v.x[2 * (e % 4) + 1] = q * t.x + p * t.y;
                } else {
                    const float p = x.x[e], q = y.x[e];
                    x.x[e] = p * t.x - q * t.y;
                    y.x[e] = q * t.x + p * t.y;
                }
            }
        }
        store8(dst + first, x);
        store8(dst + second, y);
    }
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, bool f32, bool interleaved, hipStream_t st) {
    const int64_t tokens = (int64_t)a.B * a.N;
    const int64_t steps = (a.units + 63) / 64;   // of a wavefront that takes all heads of its token
    const int64_t split = std::clamp((int64_t)2048 / tokens, (int64_t)1, steps);
    const dim3 grid((unsigned)((a.N + kTokens - 1) / kTokens), (unsigned)a.B, (unsigned)split);
    if (f32 && interleaved) hipLaunchKernelGGL((rotary_kernel<float, true>), grid, dim3(kTokens * 64), 0, st, a);
    else if (f32) hipLaunchKernelGGL((rotary_kernel<float, false>), grid, dim3(kTokens * 64), 0, st, a);
    else if (interleaved) hipLaunchKernelGGL((rotary_kernel<uint16_t, true>), grid, dim3(kTokens * 64), 0, st, a);
    else hipLaunchKernelGGL((rotary_kernel<uint16_t, false>), grid, dim3(kTokens * 64), 0, st, a);
    return hipGetLastError();
}

}  // namespace ygg
