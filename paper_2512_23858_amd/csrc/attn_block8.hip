// Tree attention over the 8-bit block cache (include/ygg.h has the format), matrix cores throughout.
//
// For one (sequence, kv head) the N nodes x G query heads are R = N*G rows that share one stream of K/V.  Two kinds of workgroup:
//
//   blocks  the full blocks of 64 tokens, as they are stored: K and V codes go from memory to LDS by direct loads and from there as
//           operands into v_mfma_scale_f32_32x32x64_f8f6f4.  S^T = K Q^T with a lane per query row, O^T += V^T P^T.  Widening the
//           codes to bf16 would cost vector work per code and twice the LDS traffic; instead the few values on the other side are
//           split: q = hi + lo with two E4M3 values that share a power of two per row and 64 dimensions (bf16 has 8 bits of
//           significand, E4M3 four, the remainder of rounding to four fits the other four), and the softmax weights likewise with a
//           power of two per row and block.  Two products at twice the bf16 rate are the bf16 rate, and P's layout as an operand is
//           that of the scores in the accumulator, because V's tokens are stored in that order: nothing changes lanes.
//   own     the open block's rows and the tree's own keys under the ancestor mask, bf16 as they are, v_mfma_f32_32x32x16_bf16.
//
// The blocks of all sequences are laid end to end and cut into equal runs, one per workgroup of a (kv head, row tile), whatever the
// lengths; a run is served segment by segment, one for each sequence that it touches.  Every segment leaves a partial (m, l, O~) per
// row: split 0 of a sequence is its own keys, 1 + r the r-th run that touches it.  attn_combine_kernel merges them.
#include "ygg_internal.h"
#include "ygg_device.h"
#include "attn_common.h"

#include <algorithm>

namespace ygg {

using namespace attn;

namespace {

typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(4))) int i32x4;

constexpr int kT = YGG_KV_BLOCK;
constexpr int kHeadroom = 7;    // weights of a block reach 2^7 (times v_scale's significand, below 2): E4M3 ends at 448
constexpr int kRescale = 30;    // a row's reference moves when a block's maximum is this many powers of two above it

template <int DH, int NW, int RB>
struct Layout {
    static constexpr int KS = NW / RB;                    // wavefronts that share a row block deal the tiles out
    static constexpr int TILE = 2 * kT * DH;              // bytes of a tile: K's codes, then V's
    static constexpr int STAGE = KS * TILE;
    static constexpr int NSTAGE = STAGE >= 65536 ? 2 : STAGE >= 32768 ? 4 : 4;
    static constexpr int OROW = DH + 4;                   // floats of a row of O~ in LDS
    static constexpr int MERGE = NW * 32 * OROW * 4;
    static constexpr int VROW = 40;                       // bf16 of a row of V^T in LDS (32 keys)
    static constexpr int OWN = KS * DH * VROW * 2;        // own keys: V^T tiles, then parents, then masks
    static constexpr int STAT = NW * 32 * 2 * 4;          // (reference, sum) of every wavefront's rows, behind everything else
    static int own_bytes(int nodes) { return OWN + nodes * 4 + RB * 32 * ((nodes + 31) / 32) * 4; }
    static size_t smem(int nodes) {
        return (size_t)std::max(std::max(NSTAGE * STAGE, MERGE), (own_bytes(nodes) + 15) / 16 * 16) + STAT;
    }
};

__device__ __forceinline__ float other_half_max(float v) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
__device__ __forceinline__ float both_halves_sum(float v) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}
// hi + lo of four values, E4M3 each
__device__ __forceinline__ void split4(const float (&x)[4], int& hi, int& lo) {
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], hi, true);
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(hi, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(hi, true);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] - a[0], x[1] - a[1], 0, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[2] - b[0], x[3] - b[1], lo, true);
}
__device__ __forceinline__ i32x8 read_operand(const unsigned char* p) {   // the two 16-byte parts of a chunk pair, 1024 bytes apart
    const i32x4 a = *reinterpret_cast<const i32x4*>(p), b = *reinterpret_cast<const i32x4*>(p + 1024);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}
__device__ __forceinline__ float uniform_load(const float* p) {   // through the scalar cache: a vector load would wait for the tiles in flight
    return *(const __attribute__((address_space(4))) float*)(p);
}

// Partial rows of one segment: the wavefronts that share a row block merge through LDS, and the rows leave as fp16 relative to c.
template <int DH, int NW, int RB>
__device__ __forceinline__ void write_partial(const Block8Args& a, unsigned char* smem, float* stat, const f32x16 (&o)[DH / 32], float ref,
                                              float l, int b, int g, int row0, int split) {
    using Lay = Layout<DH, NW, RB>;
    constexpr int KS = Lay::KS;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n = lane & 31, half = lane >> 5;
    float* const o_s = reinterpret_cast<float*>(smem);
    __syncthreads();   // the tiles are read
#pragma unroll
    for (int d = 0; d < DH / 32; ++d)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            *reinterpret_cast<float4*>(o_s + (wave * 32 + n) * Lay::OROW + 32 * d + 8 * q + 4 * half) =
                make_float4(o[d][4 * q], o[d][4 * q + 1], o[d][4 * q + 2], o[d][4 * q + 3]);
    if (half == 0) {
        stat[(wave * 32 + n) * 2] = ref;
        stat[(wave * 32 + n) * 2 + 1] = l;
    }
    __syncthreads();
    constexpr int LPR = DH / 8;   // lanes of a row
    for (int it = tid; it < RB * 32 * LPR; it += NW * 64) {
        const int r = it / LPR, col = it % LPR;
        float m = -INFINITY, w[KS], sum = 0.f;
#pragma unroll
        for (int s = 0; s < KS; ++s) m = fmaxf(m, stat[((s * RB * 32) + r) * 2]);
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const float x = stat[((s * RB * 32) + r) * 2];
            w[s] = x == -INFINITY ? 0.f : exp2f(x - m);
            sum = fmaf(stat[((s * RB * 32) + r) * 2 + 1], w[s], sum);
        }
        float v[8] = {};
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const float4* p = reinterpret_cast<const float4*>(o_s + (s * RB * 32 + r) * Lay::OROW + 8 * col);
            const float4 x = p[0], y = p[1];
            const float e[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = w[s] != 0.f ? fmaf(e[k], w[s], v[k]) : v[k];
        }
        float c = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) c = fmaxf(c, fabsf(v[k]));
        c = fmaxf(group_reduce(c, LPR, [](float x, float y) { return fmaxf(x, y); }), 1.17549435e-38f);
        const int row = row0 + r;
        if (row >= a.R) continue;
        const int node = row / a.G, h = g * a.G + row % a.G;
        const int64_t at = (int64_t)split * a.rows_total + ((int64_t)b * a.N + node) * a.Hq + h;
        __attribute__((ext_vector_type(8))) _Float16 half8;
        const float inv = 1.f / c;
#pragma unroll
        for (int k = 0; k < 8; ++k) half8[k] = (_Float16)(v[k] * inv);
        *reinterpret_cast<decltype(half8)*>(static_cast<_Float16*>(a.part_o) + at * DH + 8 * col) = half8;
        if (col == 0) a.part_rec[at] = make_float3(m, sum, c);
    }
    __syncthreads();   // before the next segment's tiles
}

__device__ __forceinline__ int length_of(const Block8Args& a, int b) {
    const int L = a.seq_lens[b];
    return L < 0 ? 0 : (L > a.max_seq_len ? a.max_seq_len : L);
}

template <int DH, int NW, int RB>
__device__ void own_keys(const Block8Args& a, unsigned char* smem, float* stat, int b, int g, int row0) {
    using Lay = Layout<DH, NW, RB>;
    constexpr int KS = Lay::KS, NK = DH / 16, NDB = DH / 32;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 31, half = lane >> 5;
    const int rb = wave % RB, share = wave / RB;
    const int L = length_of(a, b), open = L % kT;
    uint16_t* const vt = reinterpret_cast<uint16_t*>(smem) + share * DH * Lay::VROW;
    int32_t* const parent_s = reinterpret_cast<int32_t*>(smem + Lay::OWN);
    const int words = (a.N + 31) / 32;
    uint32_t* const mask_s = reinterpret_cast<uint32_t*>(parent_s + a.N) + rb * 32 * words;   // [word][row of the row block]

    const int row = min(row0 + rb * 32 + n, a.R - 1);
    const int node = row / a.G, h = g * a.G + row % a.G;
    i32x4 q[NK];
    const uint16_t* const qp = static_cast<const uint16_t*>(a.q) + (((int64_t)b * a.N + node) * a.Hq + h) * DH + 8 * half;
#pragma unroll
    for (int k = 0; k < NK; ++k) q[k] = *reinterpret_cast<const i32x4*>(qp + 16 * k);
    for (int j = tid; j < a.N; j += NW * 64) parent_s[j] = a.parent_idx[(int64_t)b * a.N + j];
    if (share == 0)
        for (int w = lane; w < 32 * words; w += 64) mask_s[w] = 0;
    __syncthreads();
    if (share == 0 && half == 0)   // a lane per row; a parent that is no earlier node ends the walk
        for (int j = node;;) {
            mask_s[(j >> 5) * 32 + n] |= 1u << (j & 31);
            const int p = parent_s[j];
            if (p < 0 || p >= j) break;
            j = p;
        }
    __syncthreads();

    const int open_tiles = (open + 31) / 32, tree_tiles = (a.N + 31) / 32, tiles = open_tiles + tree_tiles;
    const int64_t row_e = (int64_t)a.Hkv * DH;
    const int64_t first = L / kT % 2 * kT;
    const uint16_t* const kt = static_cast<const uint16_t*>(a.k_tail) + ((int64_t)b * 2 * kT + first) * row_e + (int64_t)g * DH;
    const uint16_t* const vtail = static_cast<const uint16_t*>(a.v_tail) + ((int64_t)b * 2 * kT + first) * row_e + (int64_t)g * DH;
    const uint16_t* const ktree = static_cast<const uint16_t*>(a.k_tree) + (int64_t)b * a.N * row_e + (int64_t)g * DH;
    const uint16_t* const vtree = static_cast<const uint16_t*>(a.v_tree) + (int64_t)b * a.N * row_e + (int64_t)g * DH;
    const float scale = a.scale * kLog2e;

    f32x16 o[NDB];
#pragma unroll
    for (int d = 0; d < NDB; ++d) o[d] = f32x16{};
    float m = -INFINITY, l = 0.f;
    for (int it = 0; it < tiles; it += KS) {
        const int tile = it + share;
        const bool in_tree = tile >= open_tiles;
        const int k0 = in_tree ? (tile - open_tiles) * 32 : tile * 32;
        const int valid = tile < tiles ? min(32, (in_tree ? a.N : open) - k0) : 0;   // keys of this tile
        const uint16_t* const kp = (in_tree ? ktree : kt) + (int64_t)k0 * row_e;
        const uint16_t* const vp = (in_tree ? vtree : vtail) + (int64_t)k0 * row_e;
        if (it > 0) __syncthreads();   // the previous V^T is read
        if (valid > 0) {
            // V^T by scalars: eight dimensions of a key at a time; keys beyond the last are zeros (0 * what lies there need not be 0)
            for (int p = rb * 64 + lane; p < 32 * DH / 8; p += RB * 64) {
                const int key = p % 32, d = p / 32 * 8;
                i16x8 x = {};
                if (key < valid) x = *reinterpret_cast<const i16x8*>(vp + key * row_e + d);
#pragma unroll
                for (int e = 0; e < 8; ++e) vt[(d + e) * Lay::VROW + key] = (uint16_t)x[e];
            }
        }
        __syncthreads();
        if (valid <= 0) continue;
        f32x16 s = {};
        const uint16_t* const key = kp + (int64_t)min(n, valid - 1) * row_e + 8 * half;
#pragma unroll
        for (int k = 0; k < NK; ++k)
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(key + 16 * k), __builtin_bit_cast(bf16x8, q[k]), s, 0, 0, 0);
        const uint32_t seen = in_tree ? mask_s[(k0 >> 5) * 32 + n] : valid == 32 ? 0xffffffffu : (1u << valid) - 1u;
        float top = -INFINITY;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int at = 8 * (e / 4) + 4 * half + e % 4;
            s[e] = (seen >> at) & 1u ? s[e] * scale : -INFINITY;
            top = fmaxf(top, s[e]);
        }
        top = other_half_max(top);
        const float now = fmaxf(m, top);
        const float fix = now == -INFINITY ? 1.f : exp2f(m - now);
        const float off = now == -INFINITY ? 0.f : now;
        m = now;
        l *= fix;
#pragma unroll
        for (int d = 0; d < NDB; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[d][e] *= fix;
        float p[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            p[e] = exp2f(s[e] - off);
            l += p[e];
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {   // 16 keys: 16k + 4*half + {0..3, 8..11}; weights rounded to bf16 for the product
            u32x4 w;
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = pack_bf16x2(p[8 * k + 2 * e], p[8 * k + 2 * e + 1]);
#pragma unroll
            for (int d = 0; d < NDB; ++d) {
                const uint16_t* const v = vt + (32 * d + n) * Lay::VROW + 16 * k + 4 * half;
                const u32x2 x = *reinterpret_cast<const u32x2*>(v), y = *reinterpret_cast<const u32x2*>(v + 8);
                const u32x4 operand = {x[0], x[1], y[0], y[1]};
                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, operand), __builtin_bit_cast(bf16x8, w), o[d], 0, 0, 0);
            }
        }
    }
    l = both_halves_sum(l);
    write_partial<DH, NW, RB>(a, smem, stat, o, m, l, b, g, row0, 0);
}

template <int DH, int NW, int RB>
__device__ void cache_blocks(const Block8Args& a, unsigned char* smem, float* stat, int b, int g, int row0, int t0, int t1, int split) {
    using Lay = Layout<DH, NW, RB>;
    constexpr int KS = Lay::KS, J = DH / 64, NDB = DH / 32;
    constexpr int LOADS = Lay::TILE / 1024 / RB;   // direct loads of a wavefront for its share of a tile
    constexpr int AHEAD = Lay::NSTAGE - 1;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 31, half = lane >> 5;
    const int rb = wave % RB, share = wave / RB;

    // Q: this lane's row, dimensions 64 j + 32 half .. + 31
    const int row = min(row0 + rb * 32 + n, a.R - 1);
    const int node = row / a.G, h = g * a.G + row % a.G;
    const uint16_t* const qp = static_cast<const uint16_t*>(a.q) + (((int64_t)b * a.N + node) * a.Hq + h) * DH + 32 * half;
    i32x8 qhi[J], qlo[J];
    int qscale[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
        u32x4 raw[4];
        float top = 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            raw[k] = *reinterpret_cast<const u32x4*>(qp + 64 * j + 8 * k);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                top = fmaxf(top, fmaxf(fabsf(__uint_as_float(raw[k][e] << 16)), fabsf(__uint_as_float(raw[k][e] & 0xffff0000u))));
        }
        top = other_half_max(top);
        // the largest magnitude lands in [128, 256)
        const int up = min(kHeadroom + 127 - (int)(__float_as_uint(top) >> 23), 126);
        const float by = __uint_as_float((uint32_t)(up + 127) << 23);
        qscale[j] = 127 - up;
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint32_t u = raw[k][2 * e], v = raw[k][2 * e + 1];
                const float x[4] = {__uint_as_float(u << 16) * by, __uint_as_float(u & 0xffff0000u) * by, __uint_as_float(v << 16) * by,
                                    __uint_as_float(v & 0xffff0000u) * by};
                int hi, lo;
                split4(x, hi, lo);
                qhi[j][2 * k + e] = hi;
                qlo[j][2 * k + e] = lo;
            }
    }

    const int64_t stream = ((int64_t)b * a.Hkv + g) * a.nblk;
    const int tiles = t1 - t0, steps = (tiles + KS - 1) / KS;
    const unsigned char* const kc = static_cast<const unsigned char*>(a.k_codes) + stream * kT * DH;
    const unsigned char* const vc = static_cast<const unsigned char*>(a.v_codes) + stream * kT * DH;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
    auto fill = [&](int step) {   // this wavefront's loads of its share's tile; beyond the last tile that one again, so that counts stay
        const int t = t0 + min(step * KS + share, tiles - 1);
        const unsigned char* const kb = kc + (int64_t)t * kT * DH;
        const unsigned char* const vb = vc + (int64_t)t * kT * DH;
        const uint32_t to = lds0 + (step % Lay::NSTAGE) * Lay::STAGE + share * Lay::TILE;
#pragma unroll
        for (int c = 0; c < LOADS; ++c) {
            const int chunk = rb * LOADS + c;   // K's chunks, then V's
            const unsigned char* const src = chunk < kT * DH / 1024 ? kb + chunk * 1024 : vb + (chunk - kT * DH / 1024) * 1024;
            dma_load16<false, 0>(src, (uint32_t)lane * 16, to + chunk * 1024);
        }
    };
    dma_wait_keep<0>();
    for (int s = 0; s < AHEAD; ++s) fill(s);

    f32x16 o[NDB];
#pragma unroll
    for (int d = 0; d < NDB; ++d) o[d] = f32x16{};
    int ref = 0;
    float l = 0.f;
    bool any = false;
    const float scale = a.scale * kLog2e;
    for (int step = 0; step < steps; ++step) {
        const int t = t0 + step * KS + share;
        const bool mine = t < t1;
        const float ks = uniform_load(a.k_scale + stream + min(t, t1 - 1)), vs = uniform_load(a.v_scale + stream + min(t, t1 - 1));
        dma_wait_keep<(AHEAD - 1) * LOADS>();
        lds_barrier();
        fill(step + AHEAD);
        if (!mine) continue;
        const unsigned char* const tile = smem + (step % Lay::NSTAGE) * Lay::STAGE + share * Lay::TILE + lane * 16;
        f32x16 s[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            s[u] = f32x16{};
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const i32x8 k = read_operand(tile + (u * J + j) * 2048);
                s[u] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k, qhi[j], s[u], 0, 0, 0, 127, 0, qscale[j]);
                s[u] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k, qlo[j], s[u], 0, 0, 0, 127, 0, qscale[j]);
            }
        }
        float top = -INFINITY;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, s[u][e]);
        top = other_half_max(top);
        const float by = ks * scale;
        const int c = (int)ceilf(top * by) - kHeadroom;
        if (!any) ref = c;
        any = true;
        if (__any(c - ref > kRescale)) {
            const int up = max(c - ref, 0);
            const float fix = ldexpf(1.f, -up);
            ref += up;
            l *= fix;
#pragma unroll
            for (int d = 0; d < NDB; ++d)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[d][e] *= fix;
        }
        // v_scale = significand * 2^ve: the significand joins the weights, the power is V's block scale
        const uint32_t vb = __float_as_uint(vs);
        const int ve = (int)(vb >> 23) & 255;
        const float significand = __uint_as_float((vb & 0x7fffffu) | 0x3f800000u);
        const float off = __builtin_amdgcn_logf(significand) - (float)c;
        const int pscale = max(c - ref + 127, 0);
        i32x8 phi, plo;
        float sum = 0.f;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float p[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    p[e] = __builtin_amdgcn_exp2f(fmaf(s[u][4 * q + e], by, off));
                    sum += p[e];
                }
                int hi, lo;
                split4(p, hi, lo);
                phi[4 * u + q] = hi;
                plo[4 * u + q] = lo;
            }
        l = fmaf(sum, ldexpf(1.f / significand, max(c - ref, -127)), l);
#pragma unroll
        for (int d = 0; d < NDB; ++d) {
            const i32x8 v = read_operand(tile + kT * DH + d * 2048);
            o[d] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(v, phi, o[d], 0, 0, 0, ve, 0, pscale);
            o[d] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(v, plo, o[d], 0, 0, 0, ve, 0, pscale);
        }
    }
    dma_wait_keep<0>();
    l = both_halves_sum(l);
    write_partial<DH, NW, RB>(a, smem, stat, o, any ? (float)ref : -INFINITY, l, b, g, row0, split);
}

template <int DH, int NW, int RB>
__global__ __launch_bounds__(NW * 64, NW / 4) void attn_block8_kernel(Block8Args a) {
    extern __shared__ __align__(16) unsigned char smem[];
    float* const stat = reinterpret_cast<float*>(smem + a.stat_at);
    // a stream's row tiles share an XCD, and so an L2: workgroup -> XCD is round robin
    const int xcd = blockIdx.x % 8, rest = blockIdx.x / 8;
    const int row0 = rest % a.row_tiles * RB * 32;
    const int stream = rest / a.row_tiles * 8 + xcd;
    const int own = a.B * a.Hkv;
    if (stream >= own + a.runs * a.Hkv) return;
    if (stream < own) {
        own_keys<DH, NW, RB>(a, smem, stat, stream / a.Hkv, stream % a.Hkv, row0);
        return;
    }
    const int run = (stream - own) / a.Hkv, g = (stream - own) % a.Hkv;
    int64_t total = 0;
    for (int b = 0; b < a.B; ++b) total += length_of(a, b) / kT;
    const int64_t per = max((total + a.runs - 1) / a.runs, (int64_t)1);
    const int64_t r0 = run * per, r1 = min(r0 + per, total);
    int64_t at = 0;
    for (int b = 0; b < a.B; ++b) {
        const int blocks = length_of(a, b) / kT;
        // the run that writes how many splits a sequence has: its first kv head's and row tile's run 0
        if (run == 0 && g == 0 && row0 == 0 && threadIdx.x == 0)
            a.seq_splits[b] = 1 + (blocks ? (int)((at + blocks - 1) / per - at / per + 1) : 0);
        const int64_t s0 = max(r0, at), s1 = min(r1, at + blocks);
        if (s0 < s1) cache_blocks<DH, NW, RB>(a, smem, stat, b, g, row0, (int)(s0 - at), (int)(s1 - at), 1 + (int)(run - at / per));
        at += blocks;
    }
}

template <int DH, int NW, int RB>
hipError_t raise(int) {
    return hipFuncSetAttribute(reinterpret_cast<const void*>(&attn_block8_kernel<DH, NW, RB>), hipFuncAttributeMaxDynamicSharedMemorySize,
                               (int)kAttnMfmaMaxSmem);
}

template <int DH, int NW, int RB>
hipError_t launch(Block8Args a, hipStream_t st) {
    const size_t smem = Layout<DH, NW, RB>::smem(a.N);
    if (smem > kAttnMfmaMaxSmem) return hipErrorInvalidValue;
    a.stat_at = (int32_t)(smem - Layout<DH, NW, RB>::STAT);
    const int64_t streams = (int64_t)a.B * a.Hkv + (int64_t)a.runs * a.Hkv;
    const dim3 grid((unsigned)((streams + 7) / 8 * 8 * a.row_tiles));
    hipLaunchKernelGGL((attn_block8_kernel<DH, NW, RB>), grid, dim3(NW * 64), smem, st, a);
    return hipGetLastError();
}

}  // namespace

hipError_t raise_limits_attn_block8() {
    hipError_t e = hipSuccess;
    for (hipError_t x : {raise<128, 8, 8>(0), raise<128, 8, 4>(0), raise<128, 8, 2>(0), raise<128, 4, 1>(0), raise<64, 8, 8>(0),
                         raise<64, 8, 4>(0), raise<64, 8, 2>(0), raise<64, 4, 1>(0)})
        if (x != hipSuccess) e = x;
    return e;
}

hipError_t launch_attn_block8(const Block8Args& a, const Block8Plan& p, int head_dim, hipStream_t st) {
    auto go = [&](auto dh) {
        constexpr int DH = decltype(dh)::value;
        switch (p.row_blocks) {
            case 1: return launch<DH, 4, 1>(a, st);
            case 2: return launch<DH, 8, 2>(a, st);
            case 4: return launch<DH, 8, 4>(a, st);
            default: return launch<DH, 8, 8>(a, st);
        }
    };
    return head_dim == 128 ? go(std::integral_constant<int, 128>{}) : go(std::integral_constant<int, 64>{});
}

}  // namespace ygg
