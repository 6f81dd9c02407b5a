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
// block_merge_kernel merges them.  Where that ends sooner each sequence is a workgroup's instead (plan_block).
//
// Bounds and figures: few rows are bound by the stream of codes, many by the matrix pipe and the weights' vector work beside it.  One
// token for 16 requests of 512 to 8192 tokens, 8 kv heads of 4 queries: 35.5 us with the merge, 4.0 TB/s (the main kernel 31.4, 4.5 TB/s).
// 49 rows behind 8 x 4096 tokens on 32 kv heads: 58.0 us, 4.9 TB/s.  1284 rows behind 32768 tokens: 160 to 177 us with the box's clock,
// 0.97 to 1.08 PFLOP/s counted once (each product is two on the matrix pipe).  Row blocks to a workgroup: a tile in LDS serves all of
// them, so as many as there are, up to eight; wavefronts that share a row block deal the tiles out.  One row block: two workgroups of two
// wavefronts to a compute unit 40.5 us, one of four 43.7 (one token, 16 requests).
#include "attn_block.h"

namespace ygg {
namespace {

__device__ __forceinline__ i32x8 read_operand(const unsigned char* p) {   // the two 16-byte parts of a chunk pair, 1024 bytes apart
    const i32x4 a = *reinterpret_cast<const i32x4*>(p), b = *reinterpret_cast<const i32x4*>(p + 1024);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}
__device__ __forceinline__ float uniform_load(const float* p) {   // through the scalar cache: a vector load would wait for the tiles in flight
    return *(const __attribute__((address_space(4))) float*)(p);
}

// Blocks t0 .. t1 - 1 of one stream.
template <int DH, int NW, int RB, bool NT>
__device__ __forceinline__ void cache_blocks8(unsigned char* smem, Rows<DH>& x, int b, int g, int row0, int t0, int t1) {
    Args& a = arguments();
    using Lay = Layout<8, DH, NW, RB>;
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
    const float *const ksp = static_cast<const float*>(a.k_scale) + stream, *const vsp = static_cast<const float*>(a.v_scale) + stream;
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

template <int DH, int NW, int RB, bool NT>
struct CacheBlocks<8, DH, NW, RB, NT> {
    static __device__ __forceinline__ void run(unsigned char* smem, Rows<DH>& x, int b, int g, int row0, int t0, int t1) {
        cache_blocks8<DH, NW, RB, NT>(smem, x, b, g, row0, t0, t1);
    }
};

}  // namespace

hipError_t raise_limits_attn_block8() {
    const hipError_t e = raise_for<8, 128>(), f = raise_for<8, 64>();
    return e != hipSuccess ? e : f;
}

hipError_t launch_attn_block8(const BlockArgs& a, const BlockPlan& p, int head_dim, hipStream_t st) {
    return head_dim == 128 ? launch_for<8, 128>(a, p, st) : launch_for<8, 64>(a, p, st);
}

}  // namespace ygg
