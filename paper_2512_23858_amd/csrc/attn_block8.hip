// Tree attention over the 8-bit block cache (include/ygg.h has the format), matrix cores throughout.
//
// For one (sequence, kv head) the N nodes x G query heads are R = N*G rows that share one stream of K/V.  Two kinds of keys:
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
// lengths, with room for each sequence's own keys behind its blocks; a run is served segment by segment, one for each sequence that it
// touches.  A segment that is all of its sequence writes the final rows; others leave a partial (m, l, O~) per row, and
// block8_merge_kernel merges them.  Where that ends sooner each sequence is a workgroup's instead (plan_block8).
//
// Bounds and figures: few rows are bound by the stream of codes, many by the matrix pipe and the weights' vector work beside it.  One
// token for 16 requests of 512 to 8192 tokens, 8 kv heads of 4 queries: 35.5 us with the merge, 4.0 TB/s (the main kernel 31.4, 4.5 TB/s).
// 49 rows behind 8 x 4096 tokens on 32 kv heads: 57.7 us, 4.9 TB/s.  1284 rows behind 32768 tokens: 160 to 177 us with the box's clock,
// 0.97 to 1.08 PFLOP/s counted once (each product is two on the matrix pipe).  Row blocks to a workgroup: a tile in LDS serves all of
// them, so as many as there are, up to eight; wavefronts that share a row block deal the tiles out.  One row block: two workgroups of two
// wavefronts to a compute unit 40.5 us, one of four 43.7 (one token, 16 requests).
#include "ygg_internal.h"
#include "ygg_device.h"
#include "attn_common.h"

#include <algorithm>

namespace ygg {

using namespace attn;

namespace {

typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;

constexpr int kT = YGG_KV_BLOCK;
constexpr int kHeadroom = 7;    // weights of a block reach 2^7 (times v_scale's significand, below 2): E4M3 ends at 448
constexpr int kRescale = 30;    // a row's reference moves when a block's maximum is this many powers of two above it

template <int DH, int NW, int RB>
struct Layout {
    static constexpr int KS = NW / RB;                    // wavefronts that share a row block deal the tiles out
    static constexpr int HALF = kT * DH;                  // bytes of a tile's K (or V): 64 rows of codes, or 32 of bf16
    static constexpr int CHUNKS = HALF / 1024;            // a direct load of a wavefront brings 1024 bytes
    static constexpr int LOADS = 2 * CHUNKS / RB;         // direct loads of a wavefront per tile
    static constexpr int STAGE = KS * 2 * HALF;           // [share][K, V]
    static constexpr int NSTAGE = 2;
    static constexpr int OROW = DH + 4;                   // floats of a row of O~ in LDS
    static constexpr int MERGE = NW * 32 * OROW * 4;      // in the tiles' place
    static constexpr int STAT = NW * 32 * 2 * 4;          // (reference, sum) of every wavefront's rows, behind everything else
    static constexpr int TREE = NSTAGE * STAGE;           // parents, then masks, behind the tiles
    static size_t smem(int nodes) {
        const int tree = TREE + nodes * 4 + RB * 32 * ((nodes + 31) / 32) * 4;
        return (size_t)(std::max(MERGE, tree) + 15) / 16 * 16 + STAT;
    }
};

// What a workgroup accumulates for its rows: 2^ref * O~ and 2^ref * l.  A lane holds row n = lane % 32 of its wavefront's block; ref is
// a whole number, the same in both halves of the wavefront, and l is that half's share.  A row that has seen no key yet has no reference
// (any is false, and its sums are zero): no number serves for one, since scores may lie as far below it.
template <int DH>
struct Rows {
    f32x16 o[DH / 32];
    int ref;
    float l;
    bool any;       // some key was seen: ref is set
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int d = 0; d < DH / 32; ++d) o[d] = f32x16{};
        ref = 0;
        l = 0.f;
        any = false;
    }
    // c: a whole number not below the next keys' largest score (base 2), less a constant
    __device__ __forceinline__ void refer_to(int c) {
        if (__any(c - ref > kRescale)) {
            const int up = max(c - ref, 0);
            const float fix = ldexpf(1.f, -up);
            ref += up;
            l *= fix;
#pragma unroll
            for (int d = 0; d < DH / 32; ++d)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[d][e] *= fix;
        }
    }
};

// The kernel's arguments, and the lane, as a phase of a segment first sees them: left to itself the compiler forms what depends on them
// once for all segments and keeps it in registers that the phases need (43 of them spilled).
typedef const __attribute__((address_space(4))) Block8Args Args;
__device__ __forceinline__ Args& arguments() {
    Args* p = (Args*)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *p;
}
__device__ __forceinline__ int thread_index() {
    int t = threadIdx.x;
    asm volatile("" : "+v"(t));
    return t;
}

__device__ __forceinline__ float other_half_max(float v) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
__device__ __forceinline__ float both_halves_sum(float v) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}
// hi + lo of four values, E4M3 each.  A conversion writes one half of a word, so the words' old values pass through (set to nothing first,
// they would cost a move each); the asm keeps the conversions where they are written: sunk to the words' use, in the next step behind a
// branch, they keep their arguments in registers until then.
__device__ __forceinline__ void split4(const float (&x)[4], int& hi, int& lo) {
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], hi, true);
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(hi, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(hi, true);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] - a[0], x[1] - a[1], lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[2] - b[0], x[3] - b[1], lo, true);
    asm volatile("" : "+v"(hi), "+v"(lo));
}
__device__ __forceinline__ i32x8 read_operand(const unsigned char* p) {   // the two 16-byte parts of a chunk pair, 1024 bytes apart
    const i32x4 a = *reinterpret_cast<const i32x4*>(p), b = *reinterpret_cast<const i32x4*>(p + 1024);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}
__device__ __forceinline__ float uniform_load(const float* p) {   // through the scalar cache: a vector load would wait for the tiles in flight
    return *(const __attribute__((address_space(4))) float*)(p);
}

// Rows of one segment: the wavefronts that share a row block merge through LDS; then the rows leave as a partial, fp16 relative to
// their largest magnitude, or, where the segment is all of its sequence, as they are wanted.
template <int DH, int NW, int RB>
__device__ __forceinline__ void write_rows(unsigned char* smem, float* stat, Rows<DH>& x, int b, int g, int row0,
                                           int split /* -1: final */) {
    Args& a = arguments();
    using Lay = Layout<DH, NW, RB>;
    constexpr int KS = Lay::KS;
    const int tid = thread_index(), lane = tid & 63, wave = tid >> 6;
    const int n = lane & 31, half = lane >> 5;
    float* const o_s = reinterpret_cast<float*>(smem);
    const float l = both_halves_sum(x.l);
    __syncthreads();   // the tiles are read
#pragma unroll
    for (int d = 0; d < DH / 32; ++d)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            *reinterpret_cast<float4*>(o_s + (wave * 32 + n) * Lay::OROW + 32 * d + 8 * q + 4 * half) =
                make_float4(x.o[d][4 * q], x.o[d][4 * q + 1], x.o[d][4 * q + 2], x.o[d][4 * q + 3]);
    if (half == 0) {
        stat[(wave * 32 + n) * 2] = x.any ? (float)x.ref : -INFINITY;
        stat[(wave * 32 + n) * 2 + 1] = l;
    }
    __syncthreads();
    constexpr int LPR = DH / 8;   // lanes of a row
    for (int it = tid; it < RB * 32 * LPR; it += NW * 64) {
        const int r = it / LPR, col = it % LPR;
        const int row = row0 + r;
        if (row >= a.R) break;    // (a row's lanes go together)
        float m = -INFINITY, w[KS], sum = 0.f;
#pragma unroll
        for (int s = 0; s < KS; ++s) m = fmaxf(m, stat[((s * RB * 32) + r) * 2]);
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const float y = stat[((s * RB * 32) + r) * 2];
            w[s] = y == -INFINITY ? 0.f : exp2f(y - m);
            sum = fmaf(stat[((s * RB * 32) + r) * 2 + 1], w[s], sum);
        }
        float v[8] = {};
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const float4* p = reinterpret_cast<const float4*>(o_s + (s * RB * 32 + r) * Lay::OROW + 8 * col);
            const float4 y = p[0], z = p[1];
            const float e[8] = {y.x, y.y, y.z, y.w, z.x, z.y, z.z, z.w};
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = fmaf(e[k], w[s], v[k]);
        }
        const int node = row / a.G, h = g * a.G + row % a.G;
        const int64_t out_row = ((int64_t)b * a.N + node) * a.Hq + h;
        if (split < 0) {
            const float inv = 1.f / sum;
            u32x4 y;
#pragma unroll
            for (int k = 0; k < 4; ++k) y[k] = pack_bf16x2(v[2 * k] * inv, v[2 * k + 1] * inv);
            *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(a.out) + out_row * DH + 8 * col) = y;
            if (a.lse && col == 0) a.lse[out_row] = m * kLn2 + logf(sum);
        } else {
            float c = 0.f;
#pragma unroll
            for (int k = 0; k < 8; ++k) c = fmaxf(c, fabsf(v[k]));
            c = fmaxf(group_reduce(c, LPR, [](float y, float z) { return fmaxf(y, z); }), 1.17549435e-38f);
            const int64_t at = (int64_t)split * a.rows_total + out_row;
            f16x8 y;
            const float inv = 1.f / c;
#pragma unroll
            for (int k = 0; k < 8; ++k) y[k] = (_Float16)(v[k] * inv);
            *reinterpret_cast<f16x8*>(static_cast<_Float16*>(a.part_o) + at * DH + 8 * col) = y;
            if (col == 0) a.part_rec[at] = make_float3(m, sum, c);
        }
    }
    __syncthreads();   // before the next segment's tiles
}

// The open block's rows and the tree's keys under the ancestor mask, 32 to a tile: units 0 and 1 are the open block's, 2 + k the tree's
// k-th; u0 .. u1 - 1 of them.  Tiles come in by direct loads, 16-byte slots permuted
// within a row so that operand reads meet no bank twice: K slot ^ row, V slot ^ 4 (row % (DH / 32)).
template <int DH, int NW, int RB, bool NT>
__device__ __forceinline__ void own_keys(unsigned char* smem, Rows<DH>& x, int b, int g, int row0, int L, int u0, int u1) {
    Args& a = arguments();
    using Lay = Layout<DH, NW, RB>;
    constexpr int KS = Lay::KS, NK = DH / 16, NDB = DH / 32, ROWB = 2 * DH, SLOTS = ROWB / 16, RPI = 1024 / ROWB;
    const int tid = thread_index(), lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 31, half = lane >> 5;
    const int rb = wave % RB, share = wave / RB;
    const int open = L % kT;
    const bool active = row0 + rb * 32 < a.R;
    int32_t* const parent_s = reinterpret_cast<int32_t*>(smem + Lay::TREE);
    const int words = (a.N + 31) / 32;
    uint32_t* const mask_s = reinterpret_cast<uint32_t*>(parent_s + a.N) + rb * 32 * words;   // [word][row of the row block]

    // no node sees a later one: tree keys up to the row tile's last node
    const int seen_nodes = (min(row0 + RB * 32, a.R) - 1) / a.G + 1;
    const int open0 = min(u0, (open + 31) / 32), n_open = min(u1, (open + 31) / 32) - open0;
    const int tree0 = max(u0 - 2, 0), n_tree = max(min(u1 - 2, (seen_nodes + 31) / 32) - tree0, 0);
    const int tiles = n_open + n_tree, steps = (tiles + KS - 1) / KS;
    if (tiles == 0) return;
    const int64_t row_b = (int64_t)a.Hkv * ROWB;
    const int64_t open_at = ((int64_t)b * 2 * kT + L / kT % 2 * kT) * row_b + (int64_t)g * ROWB, tree_at = (int64_t)b * a.N * row_b + (int64_t)g * ROWB;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem + share * 2 * Lay::HALF;
    auto stage_of = [](int step) { return (step & (Lay::NSTAGE - 1)) * Lay::STAGE; };
    auto fill = [&](int step) {   // rows beyond the tile's last repeat it: their weights are zero, and their values finite
        const int tile = min(step * KS + share, tiles - 1);
        const bool in_tree = tile >= n_open;
        const int k0 = (in_tree ? tree0 + tile - n_open : open0 + tile) * 32, last = (in_tree ? a.N : open) - 1 - k0;
        const unsigned char* const kb = static_cast<const unsigned char*>(in_tree ? a.k_tree : a.k_tail) + (in_tree ? tree_at : open_at) + k0 * row_b;
        const unsigned char* const vb = static_cast<const unsigned char*>(in_tree ? a.v_tree : a.v_tail) + (in_tree ? tree_at : open_at) + k0 * row_b;
        const uint32_t to = lds0 + stage_of(step);
#pragma unroll
        for (int c = 0; c < Lay::LOADS; ++c) {
            const bool is_v = Lay::CHUNKS % RB == 0 ? c >= Lay::LOADS / 2 : rb >= Lay::CHUNKS;
            const int chunk = Lay::CHUNKS % RB == 0 ? c % std::max(Lay::LOADS / 2, 1) * RB + rb : rb % Lay::CHUNKS;
            const int r = chunk * RPI + lane / SLOTS, slot = lane % SLOTS;
            const int at = is_v ? slot ^ ((r & (NDB - 1)) << 2) : slot ^ (r & (SLOTS - 1));
            dma_load16_flat<false>((is_v ? vb : kb) + min(r, last) * row_b + 16 * at, to + (is_v ? Lay::HALF : 0) + chunk * 1024);
        }
    };
    __syncthreads();   // the blocks' tiles are read
    fill(0);
    const int row = min(row0 + rb * 32 + n, a.R - 1);
    const int node = row / a.G, h = g * a.G + row % a.G;
    i32x4 q[NK];
    const uint16_t* const qp = static_cast<const uint16_t*>(a.q) + (((int64_t)b * a.N + node) * a.Hq + h) * DH + 8 * half;
#pragma unroll
    for (int k = 0; k < NK; ++k) q[k] = *reinterpret_cast<const i32x4*>(qp + 16 * k);
    for (int j = tid; j < seen_nodes; j += NW * 64) parent_s[j] = a.parent_idx[(int64_t)b * a.N + j];
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
    // K operand of step k: row n, slot 2k + half; V: the transpose read gives a lane four keys of one dimension
    const int k_lane = n * ROWB, k_xor = n & (SLOTS - 1);
    const int v_row = 4 * half + ((lane & 15) >> 2);
    const int v_lane = v_row * ROWB + 8 * (lane & 3), v_pair = (lane >> 4) & 1, v_xor = (v_row & (NDB - 1)) << 1;
    const float scale = a.scale * kLog2e;
    for (int step = 0; step < steps; ++step) {
        dma_wait_keep<0>();
        __syncthreads();
        fill(step + 1);
        const int tile = step * KS + share;
        if (tile >= tiles || !active) continue;
        const bool in_tree = tile >= n_open;
        const unsigned char* const kt = smem + stage_of(step) + share * 2 * Lay::HALF;
        const unsigned char* const vt = kt + Lay::HALF;
        f32x16 s = {};
#pragma unroll
        for (int k = 0; k < NK; ++k)
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(kt + k_lane + 16 * ((2 * k + half) ^ k_xor)),
                                                        __builtin_bit_cast(bf16x8, q[k]), s, 0, 0, 0);
        const int valid = open - (open0 + tile) * 32;
        const uint32_t seen = in_tree ? mask_s[(tree0 + tile - n_open) * 32 + n] : valid >= 32 ? 0xffffffffu : (1u << valid) - 1u;
        float top = -INFINITY;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int at = 8 * (e / 4) + 4 * half + e % 4;
            s[e] = (seen >> at) & 1u ? s[e] * scale : -INFINITY;
            top = fmaxf(top, s[e]);
        }
        top = other_half_max(top);
        const bool some = top != -INFINITY;                 // a row that sees none of the tile's keys stays as it is
        const int c = some ? (int)ceilf(top) : x.ref;
        if (!x.any) x.ref = c;
        x.any |= some;
        x.refer_to(c);
        const float off = (float)x.ref;
        float p[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {   // the sum is the log-sum-exp's too, so it takes the weights before they are rounded for the product
            p[e] = __builtin_amdgcn_exp2f(s[e] - off);
            x.l += p[e];
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {   // 16 keys: 16k + 4*half + {0..3, 8..11}; weights rounded to bf16 for the product
            u32x4 w;
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = pack_bf16x2(p[8 * k + 2 * e], p[8 * k + 2 * e + 1]);
#pragma unroll
            for (int d = 0; d < NDB; ++d) {
                const unsigned char* const v = vt + v_lane + 16 * k * ROWB + 32 * ((2 * d + v_pair) ^ v_xor);
                const i16x8 operand = __builtin_shufflevector(lds_read_tr16(v), lds_read_tr16(v + 8 * ROWB), 0, 1, 2, 3, 4, 5, 6, 7);
                x.o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, operand), __builtin_bit_cast(bf16x8, w), x.o[d], 0, 0, 0);
            }
        }
    }
    dma_wait_keep<0>();
}

// Blocks t0 .. t1 - 1 of one stream.
template <int DH, int NW, int RB, bool NT>
__device__ __forceinline__ void cache_blocks(unsigned char* smem, Rows<DH>& x, int b, int g, int row0, int t0, int t1) {
    Args& a = arguments();
    using Lay = Layout<DH, NW, RB>;
    constexpr int KS = Lay::KS, J = DH / 64, NDB = DH / 32;
    constexpr int CH = Lay::CHUNKS, LOADS = Lay::LOADS;
    const int tid = thread_index(), lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 31, half = lane >> 5;
    const int rb = wave % RB, share = wave / RB;

    const int64_t stream = ((int64_t)b * a.Hkv + g) * a.nblk;
    const int tiles = t1 - t0, steps = (tiles + KS - 1) / KS;
    const bool active = row0 + rb * 32 < a.R;
    const int mine = active ? (tiles - share + KS - 1) / KS : 0;   // this share's tiles: share, share + KS, ..
    const unsigned char* const kc = static_cast<const unsigned char*>(a.k_codes) + stream * kT * DH;
    const unsigned char* const vc = static_cast<const unsigned char*>(a.v_codes) + stream * kT * DH;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem + share * 2 * Lay::HALF;
    auto stage_of = [](int step) { return (step & (Lay::NSTAGE - 1)) * Lay::STAGE; };
    auto tile_of = [&](int step) { return t0 + min(step * KS + share, tiles - 1); };   // beyond the last tile that one again: counts stay
    // A step has the scores of the next tile, the weights of its own and the product of the one before: K runs two steps ahead of V.
    auto fill = [&](int k_step, int v_step) {
        const unsigned char* const kb = kc + (int64_t)tile_of(k_step) * Lay::HALF;
        const unsigned char* const vb = vc + (int64_t)tile_of(max(v_step, 0)) * Lay::HALF;
        const uint32_t to_k = lds0 + stage_of(k_step), to_v = lds0 + stage_of(v_step) + Lay::HALF;
#pragma unroll
        for (int c = 0; c < LOADS; ++c) {
            if constexpr (CH % RB == 0) {
                const int chunk = (c % (LOADS / 2)) * RB + rb;
                if (c < LOADS / 2) dma_load16<NT, 0>(kb + chunk * 1024, (uint32_t)lane * 16, to_k + chunk * 1024);
                else dma_load16<NT, 0>(vb + chunk * 1024, (uint32_t)lane * 16, to_v + chunk * 1024);
            } else {   // twice as many wavefronts as chunks: K's, then V's
                const int chunk = rb % CH;
                dma_load16<NT, 0>((rb < CH ? kb : vb) + chunk * 1024, (uint32_t)lane * 16, (rb < CH ? to_k : to_v) + chunk * 1024);
            }
        }
    };

#pragma unroll
    for (int c = 0; c < LOADS; ++c)
        if (c * RB + rb < CH)
            dma_load16<NT, 0>(kc + (int64_t)tile_of(0) * Lay::HALF + (c * RB + rb) * 1024, (uint32_t)lane * 16, lds0 + (c * RB + rb) * 1024);
    fill(1, -1);

    // Q: this lane's row, dimensions 64 j + 32 half .. + 31.  (Its loads come behind the first fills, and so does the wait for them.)
    const int row = min(row0 + rb * 32 + n, a.R - 1);
    const int node = row / a.G, h = g * a.G + row % a.G;
    const uint16_t* const qp = static_cast<const uint16_t*>(a.q) + (((int64_t)b * a.N + node) * a.Hq + h) * DH + 32 * half;
    i32x8 qhi[J], qlo[J];
    int qscale[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
        u32x4 raw[4];
        u16x2 most = {};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            raw[k] = *reinterpret_cast<const u32x4*>(qp + 64 * j + 8 * k);
#pragma unroll
            for (int e = 0; e < 4; ++e) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, raw[k][e] & 0x7fff7fffu));   // (bits are in the magnitudes' order)
        }
        const float top = other_half_max(__uint_as_float((uint32_t)max(most[0], most[1]) << 16));
        // the largest magnitude lands in [128, 256)
        const int up = min(kHeadroom + 127 - (int)(__float_as_uint(top) >> 23), 126);
        const float by = __uint_as_float((uint32_t)(up + 127) << 23);
        qscale[j] = 127 - up;
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint32_t u = raw[k][2 * e], v = raw[k][2 * e + 1];
                const float y[4] = {__uint_as_float(u << 16) * by, __uint_as_float(u & 0xffff0000u) * by, __uint_as_float(v << 16) * by,
                                    __uint_as_float(v & 0xffff0000u) * by};
                int hi = (int)u, lo = (int)v;    // (overwritten)
                split4(y, hi, lo);
                qhi[j][2 * k + e] = hi;
                qlo[j][2 * k + e] = lo;
            }
    }

    const unsigned char* const lane_at = smem + share * 2 * Lay::HALF + lane * 16;
    auto k_at = [&](int step) { return lane_at + stage_of(step); };
    auto v_at = [&](int step) { return lane_at + stage_of(step) + Lay::HALF; };
    struct Weights {     // of a tile's 64 keys: sum of two E4M3 values, times 2^(c - ref); ve: V's power of two
        i32x8 hi, lo;
        int c, ve;
    };
    auto meet = [&] {   // a private tile needs no meeting
        if constexpr (RB > 1) lds_barrier();
        else __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
    };

    dma_wait_keep<0>();
    meet();
    const float scale = a.scale * kLog2e;
    const float *const ksp = a.k_scale + stream, *const vsp = a.v_scale + stream;
    float ks_next = uniform_load(ksp + tile_of(0)), vs_next = uniform_load(vsp + tile_of(0));
    auto advance = [&](int step, f32x16 (&s)[2], f32x16 (&next)[2], Weights& old, Weights& w) {
        dma_wait_keep<0>();
        meet();
        fill(step + 2, step);
        if (!active) return;
        const float ks = ks_next, vs = vs_next;   // requested a step ago
        ks_next = uniform_load(ksp + tile_of(step + 1));
        vs_next = uniform_load(vsp + tile_of(step + 1));
        float top = -INFINITY;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, s[u][e]);
        top = other_half_max(top);
        const bool there = step < mine;        // (uniform) beyond this share's last tile all weights are zero
        const float by = ks * scale;
        w.c = there ? (int)ceilf(top * by) - kHeadroom : x.ref;
        // The first tile's power is the reference, and also that of the weights before it: they are zeros, but their product's scale is a
        // byte whose 255 is a NaN, and old.c - x.ref has to lie in its range, -127 (clamped) to kRescale.
        if (step == 0) x.ref = old.c = w.c;
        x.refer_to(w.c);
        // v_scale = significand * 2^ve: the significand joins the weights, the power is V's block scale
        const uint32_t vb = __float_as_uint(vs);
        w.ve = (int)(vb >> 23) & 255;
        const float significand = __uint_as_float((vb & 0x7fffffu) | 0x3f800000u);
        const float off = there ? __builtin_amdgcn_logf(significand) - (float)w.c : -INFINITY;
        // 2 J products K Q of the next tile and DH / 32 products V P of the one before take turns, two matrix instructions (hi, lo) each,
        // and this tile's weights are formed between them: a matrix instruction takes as long as 16 vector ones.  The order is the
        // program's (sched_barrier): left to itself the compiler issues them in a row, and both wavefronts of a SIMD wait for the
        // matrix pipe at once and then for the vector one.
        constexpr int UNITS = 2 * J + NDB, GROUPS = 8 / UNITS;   // groups of four weights to a unit
        const unsigned char *const kp = k_at(step + 1), *const vp = v_at(step - 1);
        const int scale_old = max(old.c - x.ref + 127, 0);
        next[0] = f32x16{};
        next[1] = f32x16{};
        auto operand = [&](int unit) { return unit % 2 == 0 ? read_operand(kp + unit / 2 * 2048) : read_operand(vp + unit / 2 * 2048); };
        i32x8 op = operand(0);
        float sum = 0.f;
        static_for<0, UNITS>([&](auto unit) {
            constexpr int U = unit, I = U / 2;
            constexpr bool QK = U % 2 == 0;
            constexpr int u = I / J, j = I % J;      // K: half of the tile, 64 dimensions
            i32x8 after;
            if constexpr (U + 1 < UNITS) after = operand(U + 1);
            float p[GROUPS][4];
            if constexpr (QK) next[u] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(op, qhi[j], next[u], 0, 0, 0, 127, 0, qscale[j]);
            else x.o[I] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(op, old.hi, x.o[I], 0, 0, 0, old.ve, 0, scale_old);
#pragma unroll
            for (int k = 0; k < GROUPS; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int at = (U * GROUPS + k) * 4 + e;
                    p[k][e] = __builtin_amdgcn_exp2f(fmaf(s[at / 16][at % 16], by, off));
                }
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (QK) next[u] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(op, qlo[j], next[u], 0, 0, 0, 127, 0, qscale[j]);
            else x.o[I] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(op, old.lo, x.o[I], 0, 0, 0, old.ve, 0, scale_old);
#pragma unroll
            for (int k = 0; k < GROUPS; ++k) {
                int hi = w.hi[U * GROUPS + k], lo = w.lo[U * GROUPS + k];
                split4(p[k], hi, lo);
                w.hi[U * GROUPS + k] = hi;
                w.lo[U * GROUPS + k] = lo;
                sum += (p[k][0] + p[k][1]) + (p[k][2] + p[k][3]);
            }
            if constexpr (U + 1 < UNITS) op = after;
            __builtin_amdgcn_sched_barrier(0);
        });
        x.l = fmaf(sum, ldexpf(__builtin_amdgcn_rcpf(significand), max(w.c - x.ref, -127)), x.l);
        // the products stay in this step too, and are not moved behind the next one's branch
#pragma unroll
        for (int u = 0; u < 2; ++u) asm volatile("" : "+v"(next[u]));
#pragma unroll
        for (int d = 0; d < NDB; ++d) asm volatile("" : "+v"(x.o[d]));
    };
    f32x16 s0[2], s1[2];
    Weights w0, w1;
    w0.hi = w0.lo = w1.hi = w1.lo = i32x8{};
    w1.c = 0;    // (as x.ref: the reference of rows that no wavefront advances)
    w1.ve = 127;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        s0[u] = f32x16{};
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const i32x8 k = read_operand(k_at(0) + (u * J + j) * 2048);
            s0[u] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k, qhi[j], s0[u], 0, 0, 0, 127, 0, qscale[j]);
            s0[u] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k, qlo[j], s0[u], 0, 0, 0, 127, 0, qscale[j]);
        }
    }
    int step = 0;
    for (; step < steps; step += 2) {
        advance(step, s0, s1, w1, w0);
        if (step + 1 == steps) {   // an odd last step
            w1 = w0;
            ++step;
            break;
        }
        advance(step + 1, s1, s0, w0, w1);
    }
    dma_wait_keep<0>();
    meet();
    x.any = mine > 0;
    const int last = max(w1.c - x.ref + 127, 0);
#pragma unroll
    for (int d = 0; d < NDB; ++d) {
        const i32x8 v = read_operand(v_at(step - 1) + d * 2048);
        x.o[d] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(v, w1.hi, x.o[d], 0, 0, 0, w1.ve, 0, last);
        x.o[d] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(v, w1.lo, x.o[d], 0, 0, 0, w1.ve, 0, last);
    }
}

// The batch laid end to end, in units of a block's time: of each sequence a.lead empty units (what a segment costs beside its keys), its
// full blocks, and a.own units for the tiles of its own keys.  Run r of `runs` has the units r * per .. (r + 1) * per - 1; with runs == 0
// each sequence is a workgroup's, and run says which.
template <int DH, int NW, int RB, bool NT>
__device__ __forceinline__ void serve(const Block8Args& a, unsigned char* smem, int g, int run, int runs, int row0, int32_t* seq_splits) {
    float* const stat = reinterpret_cast<float*>(smem + a.stat_at);
    const int lane = threadIdx.x & 63;
    // runs == 0: a workgroup to each sequence, as the only run of a batch of one
    const int begin = runs == 0 ? run : 0, end = runs == 0 ? run + 1 : a.B;
    if (runs == 0) { run = 0; runs = 1; }
    auto length = [&](int b) {
        const int L = b < end ? a.seq_lens[b] : 0;
        return L < 0 ? 0 : (L > a.max_seq_len ? a.max_seq_len : L);
    };
    int L = length(begin + lane);
    int total = end - begin == 1 ? __builtin_amdgcn_readfirstlane(L) / kT : wave_sum_i32(L / kT);
    for (int b0 = begin + 64; b0 < end; b0 += 64) total += wave_sum_i32(length(b0 + lane) / kT);
    total += (end - begin) * (a.lead + a.own);
    const int per = (total + runs - 1) / runs;
    int before = 0;
    for (int b0 = begin; b0 < end; b0 += 64) {
        if (b0 > begin) L = length(b0 + lane);
        const int blocks = L / kT, units = b0 + lane < end ? a.lead + blocks + a.own : 0;
        const int sums = end - begin == 1 ? units : wave_prefix_i32(units, lane);
        const int first = before + sums - units + a.lead;            // unit of the first block
        before += __builtin_amdgcn_readlane(sums, 63);
        const int first_run = first / per, last_run = (first + blocks + a.own - 1) / per;
        if (seq_splits && threadIdx.x < 64 && units > 0) seq_splits[b0 + lane] = last_run > first_run ? last_run - first_run + 1 : 0;
        uint64_t todo = __ballot(units > 0 && run >= first_run && run <= last_run);
        while (todo) {
            const int i = __builtin_ctzll(todo);
            todo &= todo - 1;
            const int at = __builtin_amdgcn_readlane(first, i), length = __builtin_amdgcn_readlane(L, i), nb = length / kT;
            const int from = at / per, to = (at + nb + a.own - 1) / per;
            const int lo = max(run * per - at, 0), hi = min((run + 1) * per - at, nb + a.own);
            Rows<DH> x;
            x.clear();
            if (lo < nb) cache_blocks<DH, NW, RB, NT>(smem, x, b0 + i, g, row0, lo, min(hi, nb));
            if (hi > nb) own_keys<DH, NW, RB, NT>(smem, x, b0 + i, g, row0, length, max(lo - nb, 0), hi - nb);
            write_rows<DH, NW, RB>(smem, stat, x, b0 + i, g, row0, to > from ? run - from : -1);
        }
    }
}

// RB row blocks to a workgroup; the row blocks beyond the last whole tile of eight have workgroups of REM row blocks and runs of their own.
template <int DH, int NW, int RB, int REM, bool NT>
__global__ __launch_bounds__(NW * 64, NW > 2 ? 2 : 1) void attn_block8_kernel(Block8Args a) {
    extern __shared__ __align__(16) unsigned char smem[];
    // a stream's row tiles share an XCD, and so an L2: workgroup -> XCD is round robin
    const int id = blockIdx.x;
    if (REM == 0 || id < a.main_groups) {
        const int xcd = id % 8, rest = id / 8;
        const int tile = rest % a.row_tiles, stream = rest / a.row_tiles * 8 + xcd;
        if (stream >= (a.runs ? a.runs : a.B) * a.Hkv) return;
        const int run = stream / a.Hkv, g = stream % a.Hkv;
        serve<DH, NW, RB, NT>(a, smem, g, run, a.runs, tile * RB * 32, stream == 0 && tile == 0 ? a.seq_splits : nullptr);
    } else if constexpr (REM > 0) {
        const int stream = id - a.main_groups, run = stream / a.Hkv, g = stream % a.Hkv;
        serve<DH, NW, REM, NT>(a, smem, g, run, a.rem_runs, a.row_tiles * RB * 32, stream == 0 ? a.seq_splits + a.B : nullptr);
    }
}

// Merge of a row's partials: m* = max m_s, l* = sum l_s 2^(m_s - m*), O = sum O~_s c_s 2^(m_s - m*) / l*.  DH / 8 lanes to a row, and
// GRP such groups that take every GRP-th split each; eight partials of a group are requested at once.
template <int DH, int GRP>
__global__ __launch_bounds__(256) void block8_merge_kernel(Block8Args a) {
    constexpr int LPR = DH / 8, LANES = LPR * GRP, AT_ONCE = 8;
    const int b = blockIdx.y;
    const int row = blockIdx.x * (256 / LANES) + threadIdx.x / LANES, rows = a.N * a.Hq;
    if (row >= rows) return;   // (a row's lanes go together)
    const int col = threadIdx.x % LPR, grp = threadIdx.x % LANES / LPR;
    const int local = row / a.Hq * a.G + row % a.Hq % a.G;
    const int splits = a.seq_splits[local < a.main_rows ? b : a.B + b];
    if (splits == 0) return;   // final already
    const int64_t r = (int64_t)b * rows + row;
    const f16x8* const po = static_cast<const f16x8*>(a.part_o) + r * LPR + col;
    float m = -INFINITY, l = 0.f, acc[8] = {};
    for (int s0 = grp; s0 < splits; s0 += GRP * AT_ONCE) {
        float3 rec[AT_ONCE];
        f16x8 raw[AT_ONCE];
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            const int64_t s = min(s0 + u * GRP, splits - 1);
            rec[u] = a.part_rec[s * a.rows_total + r];
            raw[u] = po[s * a.rows_total * LPR];
        }
        float top = m;
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) top = fmaxf(top, rec[u].x);
        const float fix = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
        l *= fix;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] *= fix;
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            const bool there = s0 + u * GRP < splits && rec[u].x != -INFINITY;
            const float w = there ? __builtin_amdgcn_exp2f(rec[u].x - top) : 0.f;
            l = fmaf(rec[u].y, w, l);
            const float wc = w * rec[u].z;
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] = fmaf((float)raw[u][e], wc, acc[e]);
        }
        m = top;
    }
#pragma unroll
    for (int o = LPR; o < LANES; o <<= 1) {
        const float m2 = __shfl_xor(m, o), top = fmaxf(m, m2);
        const float mine = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top), other = m2 == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m2 - top);
        l = l * mine + __shfl_xor(l, o) * other;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = acc[e] * mine + __shfl_xor(acc[e], o) * other;
        m = top;
    }
    if (grp > 0) return;
    const float inv = 1.f / l;
    u32x4 y;
#pragma unroll
    for (int k = 0; k < 4; ++k) y[k] = pack_bf16x2(acc[2 * k] * inv, acc[2 * k + 1] * inv);
    static_cast<u32x4*>(a.out)[r * LPR + col] = y;
    if (a.lse && col == 0) a.lse[r] = m * kLn2 + logf(l);
}

// Up to four row blocks there is one row tile, and beyond eight there are several.
template <int RB>
constexpr bool kOneReader = RB < 8;
template <int REM>
constexpr bool kManyReaders = REM > 0;

template <int DH, int NW, int RB, int REM>
hipError_t raise() {
    auto limit = [](auto kernel) { return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)kAttnMfmaMaxSmem); };
    hipError_t e = hipSuccess, f = hipSuccess;
    if constexpr (!kManyReaders<REM>) e = limit(&attn_block8_kernel<DH, NW, RB, REM, true>);
    if constexpr (!kOneReader<RB>) f = limit(&attn_block8_kernel<DH, NW, RB, REM, false>);
    return e != hipSuccess ? e : f;
}

template <int DH, int NW, int RB, int REM>
hipError_t launch(Block8Args a, int merge_lanes, hipStream_t st) {
    size_t smem = Layout<DH, NW, RB>::smem(a.N);
    if constexpr (REM > 0) smem = std::max(smem, Layout<DH, NW, REM>::smem(a.N));
    if (smem > kAttnMfmaMaxSmem) return hipErrorInvalidValue;
    a.stat_at = (int32_t)(smem - NW * 32 * 2 * sizeof(float));
    const int64_t streams = (int64_t)(a.runs ? a.runs : a.B) * a.Hkv;
    a.main_groups = (int32_t)((streams + 7) / 8 * 8 * a.row_tiles);
    const dim3 grid((unsigned)(a.main_groups + (REM > 0 ? (a.rem_runs ? a.rem_runs : a.B) * a.Hkv : 0)));
    // the streaming hint where a workgroup is its stream's only reader
    if constexpr (!kManyReaders<REM>)
        if (kOneReader<RB> || a.row_tiles == 1) hipLaunchKernelGGL((attn_block8_kernel<DH, NW, RB, REM, true>), grid, dim3(NW * 64), smem, st, a);
    if constexpr (!kOneReader<RB>)
        if (kManyReaders<REM> || a.row_tiles > 1) hipLaunchKernelGGL((attn_block8_kernel<DH, NW, RB, REM, false>), grid, dim3(NW * 64), smem, st, a);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess || merge_lanes == 0) return e;
    constexpr int LPR = DH / 8;
    auto groups = [&](int lanes) { return dim3((unsigned)(((int64_t)a.N * a.Hq * lanes + 255) / 256), (unsigned)a.B); };
    if (merge_lanes == 64) hipLaunchKernelGGL((block8_merge_kernel<DH, 64 / LPR>), groups(64), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((block8_merge_kernel<DH, 1>), groups(LPR), dim3(256), 0, st, a);
    return hipGetLastError();
}

template <int DH>
hipError_t launch_for(const Block8Args& a, const Block8Plan& p, hipStream_t st) {
    switch (p.row_blocks * 10 + p.rem_blocks) {
        case 10: return p.wide ? launch<DH, 4, 1, 0>(a, p.merge_lanes, st) : launch<DH, 2, 1, 0>(a, p.merge_lanes, st);
        case 20: return p.wide ? launch<DH, 8, 2, 0>(a, p.merge_lanes, st) : launch<DH, 4, 2, 0>(a, p.merge_lanes, st);
        case 40: return p.wide ? launch<DH, 8, 4, 0>(a, p.merge_lanes, st) : launch<DH, 4, 4, 0>(a, p.merge_lanes, st);
        case 80: return launch<DH, 8, 8, 0>(a, p.merge_lanes, st);
        case 82: return launch<DH, 8, 8, 2>(a, p.merge_lanes, st);
        case 84: return launch<DH, 8, 8, 4>(a, p.merge_lanes, st);
        default: return hipErrorInvalidValue;
    }
}

template <int DH>
hipError_t raise_for() {
    hipError_t e = hipSuccess;
    for (hipError_t x : {raise<DH, 2, 1, 0>(), raise<DH, 4, 2, 0>(), raise<DH, 4, 4, 0>(), raise<DH, 4, 1, 0>(), raise<DH, 8, 2, 0>(),
                         raise<DH, 8, 4, 0>(), raise<DH, 8, 8, 0>(), raise<DH, 8, 8, 2>(), raise<DH, 8, 8, 4>()})
        if (x != hipSuccess) e = x;
    return e;
}

}  // namespace

hipError_t raise_limits_attn_block8() {
    const hipError_t e = raise_for<128>(), f = raise_for<64>();
    return e != hipSuccess ? e : f;
}

hipError_t launch_attn_block8(const Block8Args& a, const Block8Plan& p, int head_dim, hipStream_t st) {
    return head_dim == 128 ? launch_for<128>(a, p, st) : launch_for<64>(a, p, st);
}

}  // namespace ygg
