// What the attention over the 8-bit and the 4-bit block cache shares: shared memory, a workgroup's rows, the open block's and the tree's
// own keys, how a batch's keys are dealt out, the merge of partial results and the launches.  What differs is CacheBlocks, the loop over
// full blocks; BITS is 8 or 4.  Included by the translation unit of each.
#pragma once
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

// Shared memory of a workgroup.  A cache tile is a block's K and V as they are stored; a tile of own keys 32 rows of bf16 of each.
template <int BITS, int DH, int NW, int RB>
struct Layout {
    static constexpr int KS = NW / RB;                    // wavefronts that share a row block deal the tiles out
    static constexpr int CODES = kT * DH * BITS / 8;      // bytes of a block's K (or V)
    static constexpr int CHUNKS = CODES / 1024;           // a direct load of a wavefront brings 1024 bytes
    static constexpr int LOADS = 2 * CHUNKS / RB;         // direct loads of a wavefront per tile
    static constexpr int SCALES = BITS == 4 ? 256 : 0;    // room for its scales
    static constexpr int SHARE = 2 * CODES + 2 * SCALES;  // [K codes, V codes, K scales, V scales]
    static constexpr int STAGE = KS * SHARE;              // [share]
    static constexpr int NSTAGE = BITS == 4 && RB > 1 ? 4 : 2;
    static constexpr int HALF = kT * DH;                  // own keys: 32 rows of K (or V)
    static constexpr int OWN_CHUNKS = HALF / 1024;
    static constexpr int OWN_LOADS = 2 * OWN_CHUNKS / RB;
    static constexpr int OWN_STAGE = KS * 2 * HALF;       // [share][K, V]
    static constexpr int OWN_STAGES = RB == 1 && KS >= 4 ? 1 : 2;   // one row block has three tiles of own keys at most: one step
    static constexpr int OROW = DH + 4;                   // floats of a row of O~ in LDS
    static constexpr int MERGE = NW * 32 * OROW * 4;      // in the tiles' place
    static constexpr int STAT = NW * 32 * 2 * 4;          // (reference, sum) of every wavefront's rows, behind everything else
    static constexpr int TREE = std::max(NSTAGE * STAGE, OWN_STAGES * OWN_STAGE);   // parents, then masks, behind the tiles
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
typedef const __attribute__((address_space(4))) BlockArgs Args;
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
// Rows of one segment: the wavefronts that share a row block merge through LDS; then the rows leave as a partial, fp16 relative to
// their largest magnitude, or, where the segment is all of its sequence, as they are wanted.
template <int BITS, int DH, int NW, int RB>
__device__ __forceinline__ void write_rows(unsigned char* smem, float* stat, Rows<DH>& x, int b, int g, int row0,
                                           int split /* -1: final */) {
    Args& a = arguments();
    using Lay = Layout<BITS, DH, NW, RB>;
    constexpr int KS = Lay::KS;
    const int tid = thread_index(), lane = tid & 63, wave = tid >> 6;
    const int n = lane & 31, half = lane >> 5;
    float* const o_s = reinterpret_cast<float*>(smem);
    const float l = both_halves_sum(x.l);
    lds_barrier();   // the tiles are read  (a barrier of LDS alone: a full one would await the rows' way to memory)
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
    lds_barrier();
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
    lds_barrier();   // before the next segment's tiles
}

// The open block's rows and the tree's keys under the ancestor mask, 32 to a tile: units 0 and 1 are the open block's, 2 + k the tree's
// k-th; u0 .. u1 - 1 of them.  Tiles come in by direct loads, 16-byte slots permuted
// within a row so that operand reads meet no bank twice: K slot ^ row, V slot ^ 4 (row % (DH / 32)).
template <int BITS, int DH, int NW, int RB>
__device__ __forceinline__ void own_keys(unsigned char* smem, Rows<DH>& x, int b, int g, int row0, int L, int u0, int u1) {
    Args& a = arguments();
    using Lay = Layout<BITS, DH, NW, RB>;
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
    auto stage_of = [](int step) { return (step & 1) * Lay::OWN_STAGE; };
    auto fill = [&](int step) {   // rows beyond the tile's last repeat it: their weights are zero, and their values finite
        const int tile = min(step * KS + share, tiles - 1);
        const bool in_tree = tile >= n_open;
        const int k0 = (in_tree ? tree0 + tile - n_open : open0 + tile) * 32, last = (in_tree ? a.N : open) - 1 - k0;
        const unsigned char* const kb = static_cast<const unsigned char*>(in_tree ? a.k_tree : a.k_tail) + (in_tree ? tree_at : open_at) + k0 * row_b;
        const unsigned char* const vb = static_cast<const unsigned char*>(in_tree ? a.v_tree : a.v_tail) + (in_tree ? tree_at : open_at) + k0 * row_b;
        const uint32_t to = lds0 + stage_of(step);
#pragma unroll
        for (int c = 0; c < Lay::OWN_LOADS; ++c) {
            const bool is_v = Lay::OWN_CHUNKS % RB == 0 ? c >= Lay::OWN_LOADS / 2 : rb >= Lay::OWN_CHUNKS;
            const int chunk = Lay::OWN_CHUNKS % RB == 0 ? c % std::max(Lay::OWN_LOADS / 2, 1) * RB + rb : rb % Lay::OWN_CHUNKS;
            const int r = chunk * RPI + lane / SLOTS, slot = lane % SLOTS;
            const int at = is_v ? slot ^ ((r & (NDB - 1)) << 2) : slot ^ (r & (SLOTS - 1));
            dma_load16_flat<false>((is_v ? vb : kb) + min(r, last) * row_b + 16 * at, to + (is_v ? Lay::HALF : 0) + chunk * 1024);
        }
    };
    lds_barrier();   // the blocks' tiles are read
    fill(0);
    if (steps > 1) fill(1);
    const int row = min(row0 + rb * 32 + n, a.R - 1);
    const int node = row / a.G, h = g * a.G + row % a.G;
    i32x4 q[NK];
    const uint16_t* const qp = static_cast<const uint16_t*>(a.q) + (((int64_t)b * a.N + node) * a.Hq + h) * DH + 8 * half;
#pragma unroll
    for (int k = 0; k < NK; ++k) q[k] = *reinterpret_cast<const i32x4*>(qp + 16 * k);
    for (int j = tid; j < seen_nodes; j += NW * 64) parent_s[j] = a.parent_idx[(int64_t)b * a.N + j];
    if (share == 0)
        for (int w = lane; w < 32 * words; w += 64) mask_s[w] = 0;
    lds_barrier();
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
        if (step > 0 && step + 1 < steps) {
            lds_barrier();      // the step before this has been read
            fill(step + 1);
        }
        if (step + 1 < steps) dma_wait_keep<Lay::OWN_LOADS>(); else dma_wait_keep<0>();
        lds_barrier();
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

// The blocks t0 .. t1 - 1 of one stream: run(smem, rows, b, g, row0, t0, t1).
template <int BITS, int DH, int NW, int RB, bool NT>
struct CacheBlocks;

// The batch laid end to end, in units of a block's time: of each sequence a.lead empty units (what a segment costs beside its keys), its
// full blocks, and a.own units for the tiles of its own keys.  Run r of `runs` has the units r * per .. (r + 1) * per - 1; with runs == 0
// each sequence is a workgroup's, and run says which.
template <int BITS, int DH, int NW, int RB, bool NT>
__device__ __forceinline__ void serve(const BlockArgs& a, unsigned char* smem, int g, int run, int runs, int row0, int32_t* seq_splits) {
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
            if (lo < nb) CacheBlocks<BITS, DH, NW, RB, NT>::run(smem, x, b0 + i, g, row0, lo, min(hi, nb));
            if (hi > nb) own_keys<BITS, DH, NW, RB>(smem, x, b0 + i, g, row0, length, max(lo - nb, 0), hi - nb);
            write_rows<BITS, DH, NW, RB>(smem, stat, x, b0 + i, g, row0, to > from ? run - from : -1);
        }
    }
}

// RB row blocks to a workgroup; the row blocks beyond the last whole tile of eight have workgroups of REM row blocks and runs of their own.
template <int BITS, int DH, int NW, int RB, int REM, bool NT>
__global__ __launch_bounds__(NW * 64, NW > 2 ? 2 : 1) void attn_block_kernel(BlockArgs a) {
    extern __shared__ __align__(16) unsigned char smem[];
    // a stream's row tiles share an XCD, and so an L2: workgroup -> XCD is round robin
    const int id = blockIdx.x;
    if (REM == 0 || id < a.main_groups) {
        const int xcd = id % 8, rest = id / 8;
        const int tile = rest % a.row_tiles, stream = rest / a.row_tiles * 8 + xcd;
        if (stream >= (a.runs ? a.runs : a.B) * a.Hkv) return;
        const int run = stream / a.Hkv, g = stream % a.Hkv;
        serve<BITS, DH, NW, RB, NT>(a, smem, g, run, a.runs, tile * RB * 32, stream == 0 && tile == 0 ? a.seq_splits : nullptr);
    } else if constexpr (REM > 0) {
        const int stream = id - a.main_groups, run = stream / a.Hkv, g = stream % a.Hkv;
        serve<BITS, DH, NW, REM, NT>(a, smem, g, run, a.rem_runs, a.row_tiles * RB * 32, stream == 0 ? a.seq_splits + a.B : nullptr);
    }
}

// Merge of a row's partials: m* = max m_s, l* = sum l_s 2^(m_s - m*), O = sum O~_s c_s 2^(m_s - m*) / l*.  DH / 8 lanes to a row, and
// GRP such groups that take every GRP-th split each; eight partials of a group are requested at once.
template <int DH, int GRP>
__global__ __launch_bounds__(256) void block_merge_kernel(BlockArgs a) {
    constexpr int LPR = DH / 8, LANES = LPR * GRP, AT_ONCE = 8;
    const int b = blockIdx.y;
    const int row = blockIdx.x * (256 / LANES) + threadIdx.x / LANES, rows = a.N * a.Hq;
    if (row >= rows) return;   // (a row's lanes go together)
    const int col = threadIdx.x % LPR, grp = threadIdx.x % LANES / LPR;
    const int local = row / a.Hq * a.G + row % a.Hq % a.G;
    const int64_t r = (int64_t)b * rows + row;
    const f16x8* const po = static_cast<const f16x8*>(a.part_o) + r * LPR + col;
    const int splits = a.seq_splits[local < a.main_rows ? b : a.B + b];
    if (splits == 0) return;   // final already
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

template <int BITS, int DH, int NW, int RB, int REM>
hipError_t raise() {
    auto limit = [](auto kernel) { return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)kAttnMfmaMaxSmem); };
    hipError_t e = hipSuccess, f = hipSuccess;
    if constexpr (!kManyReaders<REM>) e = limit(&attn_block_kernel<BITS, DH, NW, RB, REM, true>);
    if constexpr (!kOneReader<RB>) f = limit(&attn_block_kernel<BITS, DH, NW, RB, REM, false>);
    return e != hipSuccess ? e : f;
}

template <int BITS, int DH, int NW, int RB, int REM>
hipError_t launch(BlockArgs a, int merge_lanes, hipStream_t st) {
    size_t smem = Layout<BITS, DH, NW, RB>::smem(a.N);
    if constexpr (REM > 0) smem = std::max(smem, Layout<BITS, DH, NW, REM>::smem(a.N));
    if (smem > kAttnMfmaMaxSmem) return hipErrorInvalidValue;
    a.stat_at = (int32_t)(smem - NW * 32 * 2 * sizeof(float));
    const int64_t streams = (int64_t)(a.runs ? a.runs : a.B) * a.Hkv;
    a.main_groups = (int32_t)((streams + 7) / 8 * 8 * a.row_tiles);
    const dim3 grid((unsigned)(a.main_groups + (REM > 0 ? (a.rem_runs ? a.rem_runs : a.B) * a.Hkv : 0)));
    // the streaming hint where a workgroup is its stream's only reader
    if constexpr (!kManyReaders<REM>)
        if (kOneReader<RB> || a.row_tiles == 1) hipLaunchKernelGGL((attn_block_kernel<BITS, DH, NW, RB, REM, true>), grid, dim3(NW * 64), smem, st, a);
    if constexpr (!kOneReader<RB>)
        if (kManyReaders<REM> || a.row_tiles > 1) hipLaunchKernelGGL((attn_block_kernel<BITS, DH, NW, RB, REM, false>), grid, dim3(NW * 64), smem, st, a);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess || merge_lanes == 0) return e;
    constexpr int LPR = DH / 8;
    auto groups = [&](int lanes) { return dim3((unsigned)(((int64_t)a.N * a.Hq * lanes + 255) / 256), (unsigned)a.B); };
    if (merge_lanes == 64) hipLaunchKernelGGL((block_merge_kernel<DH, 64 / LPR>), groups(64), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((block_merge_kernel<DH, 1>), groups(LPR), dim3(256), 0, st, a);
    return hipGetLastError();
}

template <int BITS, int DH>
hipError_t launch_for(const BlockArgs& a, const BlockPlan& p, hipStream_t st) {
    switch (p.row_blocks * 10 + p.rem_blocks) {
        case 10:
            if constexpr (BITS == 4) return p.wide ? launch<BITS, DH, 8, 1, 0>(a, p.merge_lanes, st) : launch<BITS, DH, 4, 1, 0>(a, p.merge_lanes, st);
            else return p.wide ? launch<BITS, DH, 4, 1, 0>(a, p.merge_lanes, st) : launch<BITS, DH, 2, 1, 0>(a, p.merge_lanes, st);
        case 20: return p.wide ? launch<BITS, DH, 8, 2, 0>(a, p.merge_lanes, st) : launch<BITS, DH, 4, 2, 0>(a, p.merge_lanes, st);
        case 40: return p.wide ? launch<BITS, DH, 8, 4, 0>(a, p.merge_lanes, st) : launch<BITS, DH, 4, 4, 0>(a, p.merge_lanes, st);
        case 80: return launch<BITS, DH, 8, 8, 0>(a, p.merge_lanes, st);
        case 82: return launch<BITS, DH, 8, 8, 2>(a, p.merge_lanes, st);
        case 84: return launch<BITS, DH, 8, 8, 4>(a, p.merge_lanes, st);
        default: return hipErrorInvalidValue;
    }
}

template <int BITS, int DH>
hipError_t raise_for() {
    hipError_t e = hipSuccess;
    for (hipError_t x : {raise<BITS, DH, BITS == 4 ? 8 : 2, 1, 0>(), raise<BITS, DH, 4, 2, 0>(), raise<BITS, DH, 4, 4, 0>(), raise<BITS, DH, 4, 1, 0>(),
                         raise<BITS, DH, 8, 2, 0>(), raise<BITS, DH, 8, 4, 0>(), raise<BITS, DH, 8, 8, 0>(), raise<BITS, DH, 8, 8, 2>(), raise<BITS, DH, 8, 8, 4>()})
        if (x != hipSuccess) e = x;
    return e;
}

}  // namespace
}  // namespace ygg
