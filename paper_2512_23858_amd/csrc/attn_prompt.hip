// Causal attention of prompts (include/ygg.h: ygg_prompt_attention): bf16 on the matrix cores, and fp32 on their fp32 instructions.
//
// For one (sequence, kv head) the q_len queries x G query heads are rows that read the same keys, token by token: row r is query r / G and
// head r % G.  A workgroup takes a tile of rows and the keys that its last row sees; its wavefronts own 32 rows each and share every tile
// of 64 keys through LDS.  S^T = K Q^T with a lane per row, O^T += V^T P^T, where P's layout as an operand is that of the scores in the
// accumulator.  Row tiles are dealt out by falling position in their sequence, whatever the batch, so that the long ones start first.
//
// Bounds and figures.  Long prompts are bound by the matrix pipe and, at head_dim 64, by the vector instructions beside it (an exponential
// goes with two products of 64): 8192 tokens, heads 32/8 of 128: 462 to 485 us, 1.13 to 1.19 PFLOP/s (a large library product reaches 1.24).
// Two wavefronts to a SIMD in opposite phases (256 rows) take 474 there, two workgroups that drift (128 rows) 513.  500 and 333 tokens behind 30000 and 15000, heads 64/8: 625 to
// 655 us, 27 row tiles on the 32 compute units that a kv head has, and the clock makes up for most of the five that idle (the keys of all in
// eight parts: 640).  Eight prompts of 90 to 2047 tokens, heads 12 of 64: 38.1 us, as long as the longest prompt's last rows take over their
// 32 tiles.  A short call is a start, the chain of a row tile, and a merge where the keys are in parts.
#include "attn_common.h"

#include <algorithm>

namespace ygg {
namespace {

using namespace attn;

constexpr int kKeys = 64;   // keys of a tile

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Sequence b's lengths, cut to the rows that there are.
__device__ __forceinline__ int queries_of(const PromptArgs& a, int b) {
    if (b >= a.B) return 0;
    const int first = a.q_first[b], n = a.q_len[b];
    return first < 0 || first >= a.q_rows || n < 0 ? 0 : min(n, a.q_rows - first);
}
__device__ __forceinline__ int keys_of(const PromptArgs& a, int b) {
    const int64_t first = a.k_first[b], n = a.k_len[b];
    return first < 0 || first >= a.k_rows || n < 0 ? 0 : (int)min(min(n, (int64_t)a.max_keys), a.k_rows - first);
}

__device__ __forceinline__ int wave_sum(int v) {   // over all lanes
    v += (int)row_xor<1>((uint32_t)v);
    v += (int)row_xor<2>((uint32_t)v);
    v += (int)row_xor<7>((uint32_t)v);
    v += (int)row_xor<15>((uint32_t)v);
    const auto p = __builtin_amdgcn_permlane16_swap((uint32_t)v, (uint32_t)v, false, false);
    v = (int)(p[0] + p[1]);
    const auto q = __builtin_amdgcn_permlane32_swap((uint32_t)v, (uint32_t)v, false, false);
    return uniform((int)(q[0] + q[1]));
}

// The rank-th tile of `rows` rows in the order of falling position: those that are t-th or later in their sequences number
// S(t) = sum_b max(tiles_b - t, 0), so the rank-th is t-th for the largest t with S(t) > rank.
struct Tile {
    int b, t;   // b < 0: there are not so many
};
__device__ __forceinline__ Tile find_tile(const PromptArgs& a, int rank, int rows, int lane) {
    auto tiles_of = [&](int b) { return (int)(((int64_t)queries_of(a, b) * a.G + rows - 1) / rows); };
    const int mine = tiles_of(lane);
    if (a.B == 1) {
        const int n = uniform(mine);
        return {rank < n ? 0 : -1, n - 1 - rank};
    }
    auto later = [&](int t) {
        int s = wave_sum(max(mine - t, 0));
        for (int b0 = 64; b0 < a.B; b0 += 64) s += wave_sum(max(tiles_of(b0 + lane) - t, 0));
        return s;
    };
    if (later(0) <= rank) return {-1, 0};
    int lo = 0, hi = a.most_tiles;   // S(lo) > rank >= S(hi)
    while (hi - lo > 1) {
        const int mid = lo + (hi - lo) / 2;
        if (later(mid) > rank) lo = mid;
        else hi = mid;
    }
    int left = rank - later(hi);     // of the sequences with more than lo tiles, the left-th
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        uint64_t has = __ballot((b0 ? tiles_of(b0 + lane) : mine) > lo);
        const int count = (int)__popcll(has);
        if (left >= count) { left -= count; continue; }
        for (; left > 0; --left) has &= has - 1;
        return {b0 + __builtin_ctzll(has), lo};
    }
    return {-1, 0};
}

constexpr float kCoarse = 0x1p24f;   // references from here on, in base-2 units, are whole numbers

// s * scale - against; rounded: the product is rounded first.
__device__ __forceinline__ float less(float s, float scale, float against, bool rounded) {
#pragma clang fp contract(off)
    const float product = s * scale;
    return rounded ? product - against : fmaf(s, scale, -against);
}

// Tile buffers.  Four wavefronts: so few that two workgroups have room on a compute unit at head_dim 128 (with three buffers and one workgroup
// 4096 tokens, heads 32/8, take 189 us, so 149), and three at 64.
template <int DH, bool PHASES>
constexpr int kBuffers = PHASES ? 4 : DH == 128 ? 2 : 3;

// NW wavefronts of 32 rows.  PHASES (eight wavefronts): the two wavefronts of a SIMD are held half a block apart by a barrier between any
// two phases, so that one has the matrix pipe while the other forms its weights; it takes a fourth tile buffer.  The launch bound of two wavefronts
// to a SIMD also holds where four would do with one: above 256 registers matrix results go to accumulation registers, and are copied from
// there for the vector instructions, 48 copies to 42 of these at head_dim 64 (eight prompts of 90 to 2047 tokens 41.9 us, so 38.6).
template <int DH, int NW, bool PHASES>
__global__ __launch_bounds__(NW * 64, 2) void prompt_kernel(PromptArgs a) {
    constexpr int ROWB = 2 * DH;                 // bytes of a row in LDS
    constexpr int NS = DH / 16, NDB = DH / 32;   // steps of S^T, blocks of O^T
    constexpr int SLOTS = ROWB / 16, RPI = 1024 / ROWB;   // 16-byte slots of a row; rows of a direct load
    constexpr int RW = NW * 32, TILEB = kKeys * ROWB, NBUF = kBuffers<DH, PHASES>;
    constexpr int PT = 2 * (kKeys / RPI) / NW;   // direct loads of a wavefront per tile: K's and V's in turn
    constexpr int SH = DH == 64 ? 1 : 0;         // two rows of 128 bytes lie side by side in the banks: the slots go by pairs of rows
    static_assert(RPI * NW % (SLOTS << SH) == 0 && PT % 2 == 0, "a wavefront's rows of a tile share their place in the permutation");
    extern __shared__ __align__(16) unsigned char smem[];
    unsigned char* const k_s = smem;
    unsigned char* const v_s = smem + NBUF * TILEB;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int n = lane & 31, g2 = lane >> 5;

    const int g = blockIdx.x % a.Hkv, rank = blockIdx.x / a.Hkv / a.splits, split = blockIdx.x / a.Hkv % a.splits;
    const Tile tile = find_tile(a, rank, RW, lane);
    if (tile.b < 0) return;
    const int b = uniform(tile.b), row0 = uniform(tile.t) * RW;
    const int nq = uniform(queries_of(a, b)), nk = uniform(keys_of(a, b)), past = nk - nq;
    const int q0 = a.q_first[b];
    const int64_t k0 = a.k_first[b];
    const int R = nq * a.G;

    // this lane's row; those beyond the last repeat it and are not stored
    const int row = row0 + wave * 32 + n, rc = min(row, R - 1);
    const int query = rc / a.G, head = g * a.G + (rc - query * a.G);
    const int limit = min(max(query + past + 1, 0), nk);                         // keys that it sees
    const int first_query = row0 / a.G, last_query = (min(row0 + RW, R) - 1) / a.G;
    const int clean = min(max(first_query + past + 1, 0), nk);                   // keys that every row sees
    const int end = min(max(last_query + past + 1, 0), nk);                      // .. that any does
    // .. and that any of this wavefront's does (0: it has no rows)
    const int wave_end = row0 + wave * 32 < R ? min(max(min(row0 + wave * 32 + 31, R - 1) / a.G + past + 1, 0), nk) : 0;
    const int all_tiles = (end + kKeys - 1) / kKeys;
    const int t0 = (int)((int64_t)all_tiles * split / a.splits), t1 = (int)((int64_t)all_tiles * (split + 1) / a.splits);
    const int ntiles = t1 - t0, base = t0 * kKeys;

    f32x16 o[NDB];
#pragma unroll
    for (int d = 0; d < NDB; ++d) o[d] = f32x16{};
    float ref = limit > 0 ? -INFINITY : 0.f;     // (a row that sees nothing has weights of zero to any reference)
    float l = 0.f;
    const float scale = a.scale * kLog2e;
    float most = kWeightSumLimit;                // what a lane's weights of a block may sum to without a look at the maximum

    if (ntiles > 0) {
        bf16x8 q[NS];
        const bf16x8* const qp = reinterpret_cast<const bf16x8*>(static_cast<const uint16_t*>(a.q) + (int64_t)(q0 + query) * a.q_stride + head * DH + 8 * g2);
#pragma unroll
        for (int s = 0; s < NS; ++s) q[s] = qp[2 * s];

        // Tile fills: wavefront w's i-th load of K (or V) brings rows RPI (w + i NW) .., the slots of a row permuted on the way (attn_common.h).
        // Rows beyond the last key repeat it: their weights are zero, and its values finite.
        auto uniform_ptr = [](const unsigned char* p) {
            const uint64_t v = (uint64_t)p;
            const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
            return reinterpret_cast<const unsigned char*>(((uint64_t)hi << 32) | lo);
        };
        const unsigned char* const kb = uniform_ptr(static_cast<const unsigned char*>(a.k) + (k0 * a.k_stride + g * DH) * 2);
        const unsigned char* const vb = uniform_ptr(static_cast<const unsigned char*>(a.v) + (k0 * a.v_stride + g * DH) * 2);
        const uint32_t k_tok = (uint32_t)a.k_stride * 2, v_tok = (uint32_t)a.v_stride * 2;
        const int fill_row = RPI * wave + lane / SLOTS;
        const uint32_t k_slot = 16 * ((lane % SLOTS) ^ (fill_row >> SH & (SLOTS - 1))), v_slot = 16 * ((lane % SLOTS) ^ ((fill_row >> SH & (NDB - 1)) << 2));
        const uint32_t fill_k = fill_row * k_tok + k_slot, fill_v = fill_row * v_tok + v_slot;
        const uint32_t k_lds = uniform((uint32_t)(size_t)(__attribute__((address_space(3))) void*)k_s + wave * 1024);
        auto fill = [&](auto from, auto to, int buf, int key) __attribute__((always_inline)) {
            constexpr int FROM = decltype(from)::value, TO = decltype(to)::value;
            const uint32_t dst = uniform(k_lds + buf * TILEB);
            if (key + kKeys <= nk) {
                static_for<FROM, TO>([&](auto i) {
                    constexpr int it = i / 2;
                    constexpr bool is_v = i % 2 != 0;
                    dma_load16<false, (is_v ? NBUF * TILEB : 0) + it * NW * 1024>(uniform_ptr((is_v ? vb : kb) + (int64_t)(key + it * RPI * NW) * (is_v ? v_tok : k_tok)),
                                                                                  is_v ? fill_v : fill_k, dst);
                });
            } else if (key < base + ntiles * kKeys) {
                static_for<FROM, TO>([&](auto i) {
                    constexpr int it = i / 2;
                    constexpr bool is_v = i % 2 != 0;
                    const int64_t j = min(key + fill_row + it * RPI * NW, nk - 1);
                    dma_load16_flat<false>((is_v ? vb + j * v_tok + v_slot : kb + j * k_tok + k_slot), uniform(dst + (is_v ? NBUF * TILEB : 0) + it * NW * 1024));
                });
            }
        };
        auto fill_tile = [&](int t) { if (t < ntiles) fill(IntC<0>{}, IntC<PT>{}, t % NBUF, base + t * kKeys); };

        const int j16 = lane & 15;
        const int k_lane = n * ROWB + 16 * (g2 ^ (n >> SH & 1)), k_xor = ((n >> SH & (SLOTS - 1)) >> 1) << 5;
        const int v_row = 4 * g2 + (j16 >> 2), v_lane = v_row * ROWB + 8 * (j16 & 3), v_pair = (lane >> 4) & 1, v_xor = (v_row >> SH & (NDB - 1)) << 1;
        auto read_k = [&](int buf, int half, bf16x8 (&ka)[NS]) {
            const unsigned char* const p = k_s + buf * TILEB + half * 32 * ROWB + k_lane;
#pragma unroll
            for (int s = 0; s < NS; ++s) ka[s] = *reinterpret_cast<const bf16x8*>(p + ((32 * s) ^ k_xor));
        };
        auto read_v = [&](int buf, int half, i16x8 (&va)[NDB][2]) {
            const unsigned char* const p = v_s + buf * TILEB + half * 32 * ROWB + v_lane;
#pragma unroll
            for (int d = 0; d < NDB; ++d)
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    const unsigned char* const x = p + 16 * m * ROWB + 32 * ((2 * d + v_pair) ^ v_xor);
                    va[d][m] = __builtin_shufflevector(lds_read_tr16(x), lds_read_tr16(x + 8 * ROWB), 0, 1, 2, 3, 4, 5, 6, 7);
                }
        };
        auto qk = [&](const bf16x8 (&ka)[NS], f32x16& s) {
            s = f32x16{};
#pragma unroll
            for (int k = 0; k < NS; ++k) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka[k], q[k], s, 0, 0, 0);
        };
        auto pv = [&](const i16x8 (&va)[NDB][2], const i16x8 (&p)[2]) {
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int d = 0; d < NDB; ++d)
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, va[d][m]), __builtin_bit_cast(bf16x8, p[m]), o[d], 0, 0, 0);
        };
        // Weights against a reference that moves only when a block's sum past 2^30, as in the tree's kernel: no maximum on the common path.
        // The product of score and scale is exact within the multiply-add, and a reference is such a product rounded, so the largest score is off from
        // its own reference by up to half a step of it.  From kCoarse that is a unit and more, and soon all of a row's weights are nothing, or
        // infinite: there the products are rounded as well.  Wavefronts with such a row take the path with the maximum for every block.
        auto softmax = [&](f32x16& s, i16x8 (&p)[2], int key, bool all) {
            if (__builtin_expect(!all, 0)) {
                const int left = limit - key - 4 * g2;      // this half's keys are key + 4 g2 + 8 (e / 4) + e % 4
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] = 8 * (e / 4) + e % 4 < left ? s[e] : -INFINITY;
            }
            auto weights = [&](float against, bool coarse) __attribute__((always_inline)) {
                float sum = 0.f;
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    union { bf16x2 h[4]; i16x8 v; } w;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float x = __builtin_amdgcn_exp2f(less(s[8 * m + 2 * e], scale, against, coarse));
                        const float y = __builtin_amdgcn_exp2f(less(s[8 * m + 2 * e + 1], scale, against, coarse));
                        sum += x;
                        sum += y;
                        const f32x2 xy = {x, y};
                        w.h[e] = __builtin_convertvector(xy, bf16x2);   // the value product takes them in bf16 (nearest, ties to even)
                    }
                    p[m] = w.v;
                }
                return sum;
            };
            float sum = weights(ref, false);
            if (__builtin_expect(__any(!(sum <= most)), 0)) {   // (without a reference the sum is infinite or NaN)
                float top = s[0];
#pragma unroll
                for (int e = 1; e < 16; ++e) top = fmaxf(top, s[e]);
                top *= scale;
                top = fmaxf(top, __shfl_xor(top, 32));
                const bool raise = top > ref + kRescaleGap;
                const float fix = raise ? __builtin_amdgcn_exp2f(ref - top) : 1.f;
                if (raise) ref = top;
                l *= fix;
#pragma unroll
                for (int d = 0; d < NDB; ++d)
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[d][e] *= fix;
                const bool coarse = fabsf(ref) >= kCoarse;     // (a row that has seen no key comes here again in any case)
                most = __any(coarse) ? -1.f : kWeightSumLimit;
                sum = weights(ref == -INFINITY ? 0.f : ref, coarse);
            }
            l += sum;
        };

        bf16x8 ka[NS];
        i16x8 va[NDB][2], p[2];
        f32x16 s;
        fill_tile(0);
        fill_tile(1);
        if (ntiles > 1) dma_wait_keep<PT>(); else dma_wait_keep<0>();
        lds_barrier();
        if constexpr (NBUF > 2) fill_tile(2);
        read_k(0, 0, ka);
        if constexpr (PHASES) read_v(0, 0, va);
        qk(ka, s);

        const bool late = PHASES && wave >= 4;
        auto step = [] { asm volatile("s_barrier" ::: "memory"); };
        auto await_tile = [&](int t, bool late_, bool steady) {   // tile t + 1; a late wavefront has half of its loads of tile t + 2 before it
            if (steady || t + 2 < ntiles) {
                if (late_) dma_wait_keep<PT / 2>(); else dma_wait_keep<PT>();
            } else {
                dma_wait_keep<0>();
            }
        };
        auto interleave = [&]() {   // two or four LDS reads behind each matrix instruction
            static_for<0, NS>([&](auto) {
                __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 2 * NDB * 2 / NS, 0);
            });
        };
        auto body = [&](int t, auto bufc, auto steadyc) __attribute__((always_inline)) {
            constexpr bool STEADY = decltype(steadyc)::value;     // tiles t .. t + 3 are seen by every row, t > 0
            const int buf = bufc, next = (buf + 1) % NBUF, key = base + t * kKeys;
            const bool more = STEADY || t + 1 < ntiles;
            if constexpr (PHASES) {
                auto second_half = [&] { if (STEADY || (t > 0 && t + 2 < ntiles)) fill(IntC<PT / 2>{}, IntC<PT>{}, (buf + 2) % NBUF, key + 2 * kKeys); };
                auto first_half = [&] { if (STEADY || t + 3 < ntiles) fill(IntC<0>{}, IntC<PT / 2>{}, (buf + 3) % NBUF, key + 3 * kKeys); };
                if (key >= wave_end) {   // behind the last tile that its rows see a wavefront keeps the others company
                    if (late) await_tile(t, true, STEADY);
                    step();
                    second_half();
                    if (!late) await_tile(t, false, STEADY);
                    step();
                    step();
                    first_half();
                    step();
                    return;
                }
                read_k(buf, 1, ka);
                __builtin_amdgcn_sched_barrier(0);
                softmax(s, p, key, STEADY);   // (masked without a condition in the others: with one, hundreds of registers spill)
                __builtin_amdgcn_sched_barrier(0);
                if (late) await_tile(t, true, STEADY);
                step();
                pv(va, p);
                __builtin_amdgcn_sched_barrier(0);
                second_half();
                read_v(buf, 1, va);
                qk(ka, s);
                interleave();
                __builtin_amdgcn_sched_barrier(0);
                if (!late) await_tile(t, false, STEADY);
                step();
                if (more) read_k(next, 0, ka);
                __builtin_amdgcn_sched_barrier(0);
                softmax(s, p, key + 32, STEADY);
                __builtin_amdgcn_sched_barrier(0);
                step();
                pv(va, p);
                __builtin_amdgcn_sched_barrier(0);
                first_half();
                if (more) {
                    read_v(next, 0, va);
                    qk(ka, s);
                    interleave();
                }
                __builtin_amdgcn_sched_barrier(0);
                step();
            } else {
                read_v(buf, 0, va);
                __builtin_amdgcn_sched_barrier(0);
                softmax(s, p, key, key + 32 <= clean);
                read_k(buf, 1, ka);
                __builtin_amdgcn_sched_barrier(0);
                pv(va, p);
                qk(ka, s);
                __builtin_amdgcn_sched_barrier(0);
                read_v(buf, 1, va);
                __builtin_amdgcn_sched_barrier(0);
                softmax(s, p, key + 32, key + 64 <= clean);
                if (NBUF > 2 && t + 2 < ntiles) dma_wait_keep<PT>(); else dma_wait_keep<0>();   // tile t + 1 is here, t + 2 may be under way
                lds_barrier();
                if (t + NBUF < ntiles) fill(IntC<0>{}, IntC<PT>{}, buf, key + NBUF * kKeys);
                if (more) read_k(next, 0, ka);
                __builtin_amdgcn_sched_barrier(0);
                pv(va, p);
                if (more) qk(ka, s);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        int t = 0;
        if constexpr (PHASES) {
            if (late) step();
            const int steady_end = min((clean - base) / kKeys, ntiles) - 3;   // (clean may lie below base, or beyond this part of the keys)
            while (t < ntiles) {
                body(t, t % NBUF, std::false_type{});
                ++t;
                if (t != 1) continue;
                while (t < steady_end) {
                    body(t, IntC<1>{}, std::true_type{});
                    if (++t >= steady_end) break;
                    body(t, IntC<2>{}, std::true_type{});
                    if (++t >= steady_end) break;
                    body(t, IntC<3>{}, std::true_type{});
                    if (++t >= steady_end) break;
                    body(t, IntC<0>{}, std::true_type{});
                    ++t;
                }
            }
            if (!late) step();
        } else {
            for (; t + NBUF <= ntiles; t += NBUF) static_for<0, NBUF>([&](auto i) { body(t + i, i, std::false_type{}); });
            static_for<0, NBUF - 1>([&](auto i) {
                if (t + i < ntiles) body(t + i, i, std::false_type{});
            });
        }
    }

    // lane (n, g2) holds dimensions 32 d + 8 (e / 4) + 4 g2 + e % 4 of its row; halves swapped between the two lanes of a row leave each
    // with eight consecutive ones
    const float total = l + __shfl_xor(l, 32);
    float by = total > 0.f ? 1.f / total : 0.f, top = 1.f;
    if (a.splits > 1) {   // a partial row: fp16 relative to its largest magnitude (an error of 2^-12 of that at most)
        top = 0.f;
#pragma unroll
        for (int d = 0; d < NDB; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, fabsf(o[d][e]));
        top = fmaxf(fmaxf(top, __shfl_xor(top, 32)), 0x1p-126f);   // (the smallest normal number: its reciprocal is finite)
        by = 1.f / top;
    }
    const bool there = row < R;
    const int64_t at = (int64_t)(q0 + query) * a.Hq + head;
    uint16_t* const to = a.splits > 1 ? static_cast<uint16_t*>(a.part_o) + ((int64_t)split * a.q_rows * a.Hq + at) * DH + 8 * g2
                                      : static_cast<uint16_t*>(a.out) + at * DH + 8 * g2;
#pragma unroll
    for (int d = 0; d < NDB; ++d)
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            u32x2 even, odd;
            if (a.splits > 1) {
                const f32x4 x = {o[d][8 * m] * by, o[d][8 * m + 1] * by, o[d][8 * m + 2] * by, o[d][8 * m + 3] * by};
                const f32x4 y = {o[d][8 * m + 4] * by, o[d][8 * m + 5] * by, o[d][8 * m + 6] * by, o[d][8 * m + 7] * by};
                even = __builtin_bit_cast(u32x2, __builtin_convertvector(x, f16x4));
                odd = __builtin_bit_cast(u32x2, __builtin_convertvector(y, f16x4));
            } else {
                even = u32x2{pack_bf16x2(o[d][8 * m] * by, o[d][8 * m + 1] * by), pack_bf16x2(o[d][8 * m + 2] * by, o[d][8 * m + 3] * by)};
                odd = u32x2{pack_bf16x2(o[d][8 * m + 4] * by, o[d][8 * m + 5] * by), pack_bf16x2(o[d][8 * m + 6] * by, o[d][8 * m + 7] * by)};
            }
            const auto x = __builtin_amdgcn_permlane32_swap(even[0], odd[0], false, false);
            const auto y = __builtin_amdgcn_permlane32_swap(even[1], odd[1], false, false);
            if (there) *reinterpret_cast<u32x4*>(to + 32 * d + 16 * m) = u32x4{x[0], y[0], x[1], y[1]};
        }
    if (there && g2 == 0) {
        if (a.splits > 1) a.part_rec[(int64_t)split * a.q_rows * a.Hq + at] = make_float3(total > 0.f ? ref : -INFINITY, total, top);
        else if (a.lse) a.lse[at] = total > 0.f ? ref * kLn2 + logf(total) : -INFINITY;
    }
}

// Merge of the key splits' partial rows: DH / 8 lanes to a row, workgroups dealt out as above.
template <int DH>
__global__ __launch_bounds__(256) void prompt_merge_kernel(PromptArgs a) {
    typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
    constexpr int LPR = DH / 8, ROWS = 256 / LPR;
    const int lane = threadIdx.x & 63, g = blockIdx.x % a.Hkv;
    const Tile tile = find_tile(a, blockIdx.x / a.Hkv, ROWS, lane);
    if (tile.b < 0) return;
    const int b = uniform(tile.b), R = uniform(queries_of(a, b)) * a.G, q0 = a.q_first[b];
    const int row = uniform(tile.t) * ROWS + threadIdx.x / LPR, col = threadIdx.x % LPR;
    if (row >= R) return;
    const int query = row / a.G, head = g * a.G + row % a.G;
    const int64_t at = (int64_t)(q0 + query) * a.Hq + head, rows = (int64_t)a.q_rows * a.Hq;
    constexpr int AT_ONCE = 8;   // partials requested together (one after the other, 31 of them took 28 us)
    float m = -INFINITY, l = 0.f, acc[8] = {};
    for (int s0 = 0; s0 < a.splits; s0 += AT_ONCE) {
        float3 rec[AT_ONCE];
        f16x8 raw[AT_ONCE];
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            const int64_t r = min(s0 + u, a.splits - 1) * rows + at;
            rec[u] = a.part_rec[r];
            raw[u] = *reinterpret_cast<const f16x8*>(static_cast<const _Float16*>(a.part_o) + r * DH + 8 * col);
        }
        float top = m;
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) top = fmaxf(top, rec[u].x);
        const float fix = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
        l *= fix;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] *= fix;
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {   // (a part without keys has written zeros)
            const float w = s0 + u < a.splits && rec[u].x != -INFINITY ? __builtin_amdgcn_exp2f(rec[u].x - top) : 0.f;
            l = fmaf(rec[u].y, w, l);
            const float wc = w * rec[u].z;
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] = fmaf((float)raw[u][e], wc, acc[e]);
        }
        m = top;
    }
    const float by = l > 0.f ? 1.f / l : 0.f;
    u32x4 y;
#pragma unroll
    for (int k = 0; k < 4; ++k) y[k] = pack_bf16x2(acc[2 * k] * by, acc[2 * k + 1] * by);
    *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(a.out) + at * DH + 8 * col) = y;
    if (a.lse && col == 0) a.lse[at] = l > 0.f ? m * kLn2 + logf(l) : -INFINITY;
}

// fp32: v_mfma_f32_32x32x2_f32, four wavefronts of 32 rows, tiles of 32 keys.  A lane has one value of either operand, so which two of the
// summed values a step takes is free: of the head's dimensions 8 c + 4 half + 0 .. 3 in four steps, so that K comes in reads of 16 bytes, and
// of the keys the two that a score register holds in the two halves, so that the weights are operands as they lie.  Keys are never in parts, and
// a row tile is 128 rows however few there are: 512 tokens, heads 32/8 of 128, 78 us, 2048 tokens 406, but 16 tokens behind 30000 take 4.1 ms,
// one chain of 938 tiles on eight compute units.
template <int DH>
__global__ __launch_bounds__(256, 2) void prompt_f32_kernel(PromptArgs a) {
    constexpr int KT = 32, PITCH = DH + 4, RW = 128, NDB = DH / 32, NC = DH / 8;
    __shared__ __align__(16) float k_s[KT * PITCH], v_s[KT * PITCH];
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), n = lane & 31, half = lane >> 5;
    const int g = blockIdx.x % a.Hkv;
    const Tile tile = find_tile(a, blockIdx.x / a.Hkv, RW, lane);
    if (tile.b < 0) return;
    const int b = uniform(tile.b), row0 = uniform(tile.t) * RW;
    const int nq = uniform(queries_of(a, b)), nk = uniform(keys_of(a, b)), past = nk - nq;
    const int q0 = a.q_first[b];
    const int64_t k0 = a.k_first[b];
    const int R = nq * a.G, row = row0 + wave * 32 + n, rc = min(row, R - 1);
    const int query = rc / a.G, head = g * a.G + (rc - query * a.G);
    const int limit = min(max(query + past + 1, 0), nk);
    const int end = min(max((min(row0 + RW, R) - 1) / a.G + past + 1, 0), nk);
    const int wave_end = row0 + wave * 32 < R ? min(max(min(row0 + wave * 32 + 31, R - 1) / a.G + past + 1, 0), nk) : 0;
    f32x4 q[NC];
    const f32x4* const qp = reinterpret_cast<const f32x4*>(static_cast<const float*>(a.q) + (int64_t)(q0 + query) * a.q_stride + head * DH + 4 * half);
#pragma unroll
    for (int c = 0; c < NC; ++c) q[c] = qp[2 * c];
    f32x16 o[NDB];
#pragma unroll
    for (int d = 0; d < NDB; ++d) o[d] = f32x16{};
    float ref = -INFINITY, l = 0.f;
    const float* const kb = static_cast<const float*>(a.k) + k0 * a.k_stride + g * DH;
    const float* const vb = static_cast<const float*>(a.v) + k0 * a.v_stride + g * DH;
    const float scale = a.scale * kLog2e;
    constexpr int PIECES = KT * DH / 4 / 256;   // of 16 bytes, per thread
    f32x4 kr[PIECES], vr[PIECES];
    auto request = [&](int key) {
#pragma unroll
        for (int u = 0; u < PIECES; ++u) {
            const int p = tid + 256 * u;
            const int64_t j = min(key + p / (DH / 4), nk - 1);
            kr[u] = *reinterpret_cast<const f32x4*>(kb + j * a.k_stride + 4 * (p % (DH / 4)));
            vr[u] = *reinterpret_cast<const f32x4*>(vb + j * a.v_stride + 4 * (p % (DH / 4)));
        }
    };
    if (end > 0) request(0);
    for (int key = 0; key < end; key += KT) {
        __syncthreads();
#pragma unroll
        for (int u = 0; u < PIECES; ++u) {
            const int p = tid + 256 * u, at = p / (DH / 4) * PITCH + 4 * (p % (DH / 4));
            *reinterpret_cast<f32x4*>(k_s + at) = kr[u];
            *reinterpret_cast<f32x4*>(v_s + at) = vr[u];
        }
        __syncthreads();
        if (key + KT < end) request(key + KT);
        if (key >= wave_end) continue;
        f32x16 s = {};
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const f32x4 k = *reinterpret_cast<const f32x4*>(k_s + n * PITCH + 8 * c + 4 * half);
#pragma unroll
            for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(k[e], q[c][e], s, 0, 0, 0);
        }
        const int left = limit - key - 4 * half;
        float top = -INFINITY;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            s[e] = 8 * (e / 4) + e % 4 < left ? s[e] * scale : -INFINITY;
            top = fmaxf(top, s[e]);
        }
        top = fmaxf(top, __shfl_xor(top, 32));
        if (top > ref) {
            const float fix = __builtin_amdgcn_exp2f(ref - top);
            ref = top;
            l *= fix;
#pragma unroll
            for (int d = 0; d < NDB; ++d)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[d][e] *= fix;
        }
        const float against = ref == -INFINITY ? 0.f : ref;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            s[e] = __builtin_amdgcn_exp2f(s[e] - against);
            l += s[e];
        }
#pragma unroll
        for (int e = 0; e < 16; ++e)
#pragma unroll
            for (int d = 0; d < NDB; ++d)
                o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(v_s[(8 * (e / 4) + 4 * half + e % 4) * PITCH + 32 * d + n], s[e], o[d], 0, 0, 0);
    }
    const float total = l + __shfl_xor(l, 32), by = total > 0.f ? 1.f / total : 0.f;
    if (row >= R) return;
    const int64_t at = (int64_t)(q0 + query) * a.Hq + head;
    float* const to = static_cast<float*>(a.out) + at * DH + 4 * half;
#pragma unroll
    for (int d = 0; d < NDB; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            *reinterpret_cast<f32x4*>(to + 32 * d + 8 * e) = f32x4{o[d][4 * e] * by, o[d][4 * e + 1] * by, o[d][4 * e + 2] * by, o[d][4 * e + 3] * by};
    if (a.lse && half == 0) a.lse[at] = total > 0.f ? ref * kLn2 + logf(total) : -INFINITY;
}

template <int DH, int NW, bool PHASES>
constexpr int kSmem = 2 * kBuffers<DH, PHASES> * kKeys * 2 * DH;

template <int DH, int NW, bool PHASES>
hipError_t raise() {
    return hipFuncSetAttribute(reinterpret_cast<const void*>(&prompt_kernel<DH, NW, PHASES>), hipFuncAttributeMaxDynamicSharedMemorySize, kSmem<DH, NW, PHASES>);
}

template <int DH>
hipError_t launch_for(const PromptArgs& a, const PromptPlan& p, hipStream_t st) {
    const dim3 grid((unsigned)((int64_t)p.ranks * a.Hkv * a.splits));
    if (p.waves == 8) hipLaunchKernelGGL((prompt_kernel<DH, 8, true>), grid, dim3(512), (kSmem<DH, 8, true>), st, a);
    else hipLaunchKernelGGL((prompt_kernel<DH, 4, false>), grid, dim3(256), (kSmem<DH, 4, false>), st, a);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess || a.splits == 1) return e;
    PromptArgs m = a;
    m.most_tiles = p.merge_most_tiles;
    hipLaunchKernelGGL((prompt_merge_kernel<DH>), dim3((unsigned)((int64_t)p.merge_ranks * a.Hkv)), dim3(256), 0, st, m);
    return hipGetLastError();
}

}  // namespace

hipError_t raise_limits_attn_prompt() {
    for (hipError_t e : {raise<128, 8, true>(), raise<128, 4, false>(), raise<64, 8, true>(), raise<64, 4, false>()})
        if (e != hipSuccess) return e;
    return hipSuccess;
}

hipError_t launch_attn_prompt(const PromptArgs& a, const PromptPlan& p, int head_dim, bool f32, hipStream_t st) {
    if (!f32) return head_dim == 128 ? launch_for<128>(a, p, st) : launch_for<64>(a, p, st);
    const dim3 grid((unsigned)((int64_t)p.ranks * a.Hkv));
    if (head_dim == 128) hipLaunchKernelGGL((prompt_f32_kernel<128>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((prompt_f32_kernel<64>), grid, dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace ygg
