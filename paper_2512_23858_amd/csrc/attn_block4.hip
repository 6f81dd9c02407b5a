// Tree attention over the 4-bit block cache (include/ygg.h has the format), matrix cores throughout.
//
// The rows, runs, own keys and the merge are those of the 8-bit cache (attn_block.h).  Blocks are streamed as they are stored: E2M1 codes
// are operands of v_mfma_scale_f32_32x32x64_f8f6f4 as they lie in memory, and the scale of 32 values is that instruction's own scale of a
// row's 32 values, so K's scales are part of the scores and V's of the output without a vector instruction.  q and the weights are sums of
// two E4M3 values as there: with both sides in six bits or fewer the products would take half the time, but E2M3 has no range: a weight
// 2^-8 of its tile's largest would be rounded to nothing, and 63 of those beside a large one are a tenth of a row.
// An operand in 8 bits holds its 32 values of a lane as 16 and 16 of either half of the 64 that a product sums, one in 4 bits a half as a
// whole: q is loaded to match, and V's tokens are stored to match the scores in the accumulator.
//
// Half the bytes per block of the 8-bit cache leave less in flight: where row blocks share tiles four stages of them instead of two, filled
// three steps ahead.  One row block has four wavefronts to itself and two stages: with two wavefronts and four stages 30.2 us, so 28.6, for
// one token for 16 requests of 512 to 8192 tokens, 8 kv heads of 4 queries (2.8 TB/s; 24.9 in the main kernel, bound by the latency of a
// run's start and of each segment's own keys, and the merge behind it).  49 nodes behind 8 x 16384 tokens on those heads: 120 us,
// 30 to 33 by the operations at these instructions' rate (3.2 to 3.5 PFLOP/s with random operands) and twice that for q's and the weights' two terms; bound
// by the weights' vector work, 264 instructions for a wavefront's 32 rows of a tile, which overlap with the matrix pipe (48 % busy)
// only across wavefronts.  q as two E2M3 values would take half the time on that pipe and the call 114 us, but a format of two exponent
// bits keeps what is near the largest of 32 dimensions: a q with one large dimension would lose the others' low bits.
#include "attn_block.h"

namespace ygg {
namespace {

constexpr int kE2M1 = 4;   // the matrix instruction's format code (0: E4M3)

__device__ __forceinline__ i32x8 read_operand(const unsigned char* p) {   // 32 codes; the instruction reads four registers of the eight
    const i32x4 a = *reinterpret_cast<const i32x4*>(p);
    return __builtin_shufflevector(a, a, 0, 1, 2, 3, -1, -1, -1, -1);
}

// Blocks t0 .. t1 - 1 of one stream.
template <int DH, int NW, int RB, bool NT>
__device__ __forceinline__ void cache_blocks4(unsigned char* smem, Rows<DH>& x, int b, int g, int row0, int t0, int t1) {
    Args& a = arguments();
    using Lay = Layout<4, DH, NW, RB>;
    constexpr int KS = Lay::KS, J = DH / 64, NDB = DH / 32, NS = Lay::NSTAGE, CH = Lay::CHUNKS;
    // direct loads of a wavefront per step: chunks of K and V, or one of both together where there are more wavefronts than chunks of K
    // (some then twice, with the same bytes), and scales (K's by even row blocks and V's by odd ones, likewise)
    constexpr bool FEW = CH % RB != 0;
    constexpr int LOADS = (FEW ? 1 : 2 * CH / RB) + (RB == 1 ? 2 : 1);
    const int tid = thread_index(), lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 31, half = lane >> 5;
    const int rb = wave % RB, share = wave / RB;

    const int64_t stream = ((int64_t)b * a.Hkv + g) * a.nblk;
    const int tiles = t1 - t0, steps = (tiles + KS - 1) / KS;
    const bool active = row0 + rb * 32 < a.R;
    const int mine = active ? (tiles - share + KS - 1) / KS : 0;   // this share's tiles: share, share + KS, ..
    const unsigned char* const kc = static_cast<const unsigned char*>(a.k_codes) + stream * Lay::CODES;
    const unsigned char* const vc = static_cast<const unsigned char*>(a.v_codes) + stream * Lay::CODES;
    const unsigned char* const ksp = static_cast<const unsigned char*>(a.k_scale) + stream * 2 * DH;
    const unsigned char* const vsp = static_cast<const unsigned char*>(a.v_scale) + stream * 2 * DH;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem + share * Lay::SHARE;
    auto stage_of = [](int step) { return (step & (NS - 1)) * Lay::STAGE; };
    auto tile_of = [&](int step) { return t0 + min(max(step, 0) * KS + share, tiles - 1); };   // beyond the last tile that one again: counts stay
    // A step has the scores of the next tile, the weights of its own and the product of the one before: K runs two steps ahead of V.
    auto fill = [&](int k_step) {
        const int v_step = k_step - 2;
        const int64_t kt = tile_of(k_step), vt = tile_of(v_step);
        const unsigned char* const kb = kc + kt * Lay::CODES;
        const unsigned char* const vb = vc + vt * Lay::CODES;
        const uint32_t to_k = lds0 + stage_of(k_step), to_v = lds0 + stage_of(v_step) + Lay::CODES;
        if constexpr (FEW) {
            const int chunk = rb % CH;
            const bool is_k = rb % (2 * CH) < CH;
            dma_load16<NT, 0>((is_k ? kb : vb) + chunk * 1024, (uint32_t)lane * 16, (is_k ? to_k : to_v) + chunk * 1024);
        } else {
#pragma unroll
            for (int c = 0; c < CH / RB; ++c) dma_load16<NT, 0>(kb + (c * RB + rb) * 1024, (uint32_t)lane * 16, to_k + (c * RB + rb) * 1024);
#pragma unroll
            for (int c = 0; c < CH / RB; ++c) dma_load16<NT, 0>(vb + (c * RB + rb) * 1024, (uint32_t)lane * 16, to_v + (c * RB + rb) * 1024);
        }
        const uint32_t word = (uint32_t)(lane % (DH / 2)) * 4;   // (head_dim 64: the second half of the lanes repeats the first)
        if (RB == 1 || rb % 2 == 0) dma_load4(ksp + kt * 2 * DH + word, lds0 + stage_of(k_step) + 2 * Lay::CODES);
        if (RB == 1 || rb % 2 != 0) dma_load4(vsp + vt * 2 * DH + word, lds0 + stage_of(v_step) + 2 * Lay::CODES + Lay::SCALES);
    };

    fill(0);
    fill(1);

    // Q: this lane's row, dimensions 64 j + 16 half .. + 15 and those 32 further.  (Its loads come behind the first fills, and so does the
    // wait for them.)
    const int row = min(row0 + rb * 32 + n, a.R - 1);
    const int node = row / a.G, h = g * a.G + row % a.G;
    const uint16_t* const qp = static_cast<const uint16_t*>(a.q) + (((int64_t)b * a.N + node) * a.Hq + h) * DH + 16 * half;
    i32x8 qhi[J], qlo[J];
    int qscale[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
        u32x4 raw[4];
        u16x2 most = {};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            raw[k] = *reinterpret_cast<const u32x4*>(qp + 64 * j + 32 * (k / 2) + 8 * (k % 2));
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

    static_for<2, NS>([&](auto p) { fill(p); });

    const unsigned char* const lane_at = smem + share * Lay::SHARE + lane * 16;
    auto k_at = [&](int step) { return lane_at + stage_of(step); };
    auto v_at = [&](int step) { return lane_at + stage_of(step) + Lay::CODES; };
    auto scales_of = [&](int step, int is_v) -> int {   // this lane's DH / 32 scale bytes of a tile
        const unsigned char* const p = smem + share * Lay::SHARE + stage_of(step) + 2 * Lay::CODES + is_v * Lay::SCALES + lane * (DH / 32);
        if constexpr (DH == 128) return *reinterpret_cast<const int*>(p);
        else return *reinterpret_cast<const uint16_t*>(p);
    };
    struct Weights {     // of a tile's 64 keys: sum of two E4M3 values, times 2^(c - ref)
        i32x8 hi, lo;
        int c;
    };
    auto meet = [&] {   // a private tile needs no meeting
        if constexpr (RB > 1) lds_barrier();
        else __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
    };

    dma_wait_keep<(NS - 1) * LOADS>();
    meet();
    const float scale = a.scale * kLog2e;
    auto advance = [&](int step, f32x16 (&s)[2], f32x16 (&next)[2], Weights& old, Weights& w) {
        dma_wait_keep<(NS - 2) * LOADS>();   // K of step + 1 and V of step - 1 are here, two fills may be under way
        meet();
        fill(step + NS);
        if (!active) return;
        float top = -INFINITY;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, s[u][e]);
        top = other_half_max(top);
        const bool there = step < mine;        // (uniform) beyond this share's last tile all weights are zero
        w.c = there ? (int)ceilf(top * scale) - kHeadroom : x.ref;
        // The first tile's power is the reference, and also that of the weights before it: they are zeros, but their product's scale is a
        // byte whose 255 is a NaN, and old.c - x.ref has to lie in its range, -127 (clamped) to kRescale.
        if (step == 0) x.ref = old.c = w.c;
        x.refer_to(w.c);
        const float off = there ? -(float)w.c : -INFINITY;
        // 2 J products K Q of the next tile and DH / 32 products V P of the one before take turns, two matrix instructions (hi, lo) each,
        // and this tile's weights are formed between them: a matrix instruction takes as long as 16 vector ones.  The order is the
        // program's (sched_barrier): left to itself the compiler issues them in a row, and both wavefronts of a SIMD wait for the
        // matrix pipe at once and then for the vector one.
        constexpr int UNITS = 2 * J + NDB, GROUPS = 8 / UNITS;   // groups of four weights to a unit
        const unsigned char *const kp = k_at(step + 1), *const vp = v_at(step - 1);
        const int ks = scales_of(step + 1, 0), vs = scales_of(step - 1, 1);
        const int scale_old = max(old.c - x.ref + 127, 0);
        next[0] = f32x16{};
        next[1] = f32x16{};
        auto operand = [&](int unit) { return unit % 2 == 0 ? read_operand(kp + unit / 2 * 1024) : read_operand(vp + unit / 2 * 1024); };
        i32x8 op = operand(0);
        float sum = 0.f;
        static_for<0, UNITS>([&](auto unit) {
            constexpr int U = unit, I = U / 2;
            constexpr bool QK = U % 2 == 0;
            constexpr int u = I / J, j = I % J;      // K: half of the tile, 64 dimensions
            i32x8 after;
            if constexpr (U + 1 < UNITS) after = operand(U + 1);
            float p[GROUPS][4];
            if constexpr (QK) next[u] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(op, qhi[j], next[u], kE2M1, 0, I, ks, 0, qscale[j]);
            else x.o[I] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(op, old.hi, x.o[I], kE2M1, 0, I, vs, 0, scale_old);
#pragma unroll
            for (int k = 0; k < GROUPS; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int at = (U * GROUPS + k) * 4 + e;
                    p[k][e] = __builtin_amdgcn_exp2f(fmaf(s[at / 16][at % 16], scale, off));
                }
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (QK) next[u] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(op, qlo[j], next[u], kE2M1, 0, I, ks, 0, qscale[j]);
            else x.o[I] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(op, old.lo, x.o[I], kE2M1, 0, I, vs, 0, scale_old);
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
        x.l = fmaf(sum, ldexpf(1.f, max(w.c - x.ref, -127)), x.l);
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
    const int first = scales_of(0, 0);
    s0[0] = s0[1] = f32x16{};
    static_for<0, 2 * J>([&](auto unit) {
        constexpr int I = unit, u = I / J, j = I % J;
        const i32x8 k = read_operand(k_at(0) + I * 1024);
        s0[u] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k, qhi[j], s0[u], kE2M1, 0, I, first, 0, qscale[j]);
        s0[u] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k, qlo[j], s0[u], kE2M1, 0, I, first, 0, qscale[j]);
    });
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
    const int last = max(w1.c - x.ref + 127, 0), vs = scales_of(step - 1, 1);
    static_for<0, NDB>([&](auto d) {
        const i32x8 v = read_operand(v_at(step - 1) + d * 1024);
        x.o[d] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(v, w1.hi, x.o[d], kE2M1, 0, d, vs, 0, last);
        x.o[d] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(v, w1.lo, x.o[d], kE2M1, 0, d, vs, 0, last);
    });
}

template <int DH, int NW, int RB, bool NT>
struct CacheBlocks<4, DH, NW, RB, NT> {
    static __device__ __forceinline__ void run(unsigned char* smem, Rows<DH>& x, int b, int g, int row0, int t0, int t1) {
        cache_blocks4<DH, NW, RB, NT>(smem, x, b, g, row0, t0, t1);
    }
};

}  // namespace

hipError_t raise_limits_attn_block4() {
    const hipError_t e = raise_for<4, 128>(), f = raise_for<4, 64>();
    return e != hipSuccess ? e : f;
}

hipError_t launch_attn_block4(const BlockArgs& a, const BlockPlan& p, int head_dim, hipStream_t st) {
    return head_dim == 128 ? launch_for<4, 128>(a, p, st) : launch_for<4, 64>(a, p, st);
}

}  // namespace ygg
