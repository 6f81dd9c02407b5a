// Host side of the C ABI: argument validation, launch plans, workspace carving.  No device work
// is done here other than enqueuing kernels on the caller's stream; nothing synchronises.
#include "ygg_internal.h"

#include <algorithm>
#include <atomic>
#include <cmath>
#include <mutex>
#include <type_traits>

namespace ygg {
namespace {

// Launch-plan override for tuning runs (ygg_debug_set_attention_plan): waves << 24 | rblocks << 16 | kshares << 8 in the
// upper word, the forced split count in the lower; 0 = no override.
std::atomic<uint64_t> g_plan_override{0};

// One-time set-up per device: every kernel variant that needs more dynamic shared memory than the default gets its limit
// raised, so that no later call (possibly under stream capture) has to.
constexpr int kMaxDevices = 64;
std::atomic<bool> g_device_ready[kMaxDevices];
std::mutex g_init_mutex;

// Library-owned workspace of ygg_equal_growth_expand_static, for callers that cannot provide one.  Every device
// holds its own copy at its own address (looked up once per device, below); host code only ever uses that
// address.  Nothing in it has to start at zero: every call writes what it reads.
constexpr size_t kStaticScratchBytes = YGG_STATIC_SCRATCH_BYTES;
static __device__ __align__(256) unsigned char scratch[kStaticScratchBytes];
unsigned char* g_scratch_ptr[kMaxDevices];

// What a segment of a balanced batch costs beside its key tiles (Q, masks, an empty pipeline, the partial rows), in tiles.
// us per call, 0 / 3 / 6 / 8 tiles: 16 sequences of 512 to 8192 tokens with 392 rows on 8 kv heads 165 / 157 / 152 / 149, 8 of 256 to
// 8192 with 516 rows 115 / 111 / 110 / 112, 4 of 1024 to 16384 with 196 rows 59 / 57 / 54 / 53, 40 of 100 to 3000 with 392 rows 169 /
// 165 / 159 / 156, 9 of 1 to 4000 with 164 rows 42 / 33 / 29 / 29; six equal ones of 1024 with 516 rows 41 / 39 / 40 / 41.
constexpr int32_t kSegmentLead = 6;

inline size_t align256(size_t x) { return (x + 255) / 256 * 256; }

bool common_shape_ok(const ygg_shape& s) {
    if (s.batch < 1 || s.batch > 65535) return false;
    if (s.n_q_heads < 1 || s.n_kv_heads < 1 || s.n_q_heads % s.n_kv_heads != 0) return false;
    if (s.depth < 0 || s.width < 1 || s.n_nodes < 1) return false;
    if (s.max_seq_len < 0 || s.kv_capacity < (int64_t)s.max_seq_len + s.depth + 1) return false;
    return true;
}

int32_t check_shape(const ygg_shape* s, bool need_kv, bool need_vocab) {
    if (!s) return YGG_ERR_NULL;
    if (!common_shape_ok(*s)) return YGG_ERR_SHAPE;
    if (s->n_nodes > kMaxNodes || s->width > kMaxWidth) return YGG_ERR_UNSUPPORTED;
    if (need_kv) {
        if (s->kv_dtype != YGG_F32 && s->kv_dtype != YGG_BF16 && s->kv_dtype != YGG_FP8_E4M3) return YGG_ERR_UNSUPPORTED;
        if (s->head_dim != 64 && s->head_dim != 128) return YGG_ERR_UNSUPPORTED;
        if (s->kv_dtype == YGG_FP8_E4M3 && s->head_dim != 128) return YGG_ERR_UNSUPPORTED;
        // the matrix-core kernel takes row maxima before scaling, which needs a positive finite scale
        if (!(s->softmax_scale > 0.f) || !std::isfinite(s->softmax_scale)) return YGG_ERR_SHAPE;
    }
    if (need_vocab && s->vocab < 1) return YGG_ERR_SHAPE;
    return YGG_OK;
}

// Shapes of the calls on a block cache: dtype YGG_FP8_BLOCK or YGG_FP4_BLOCK.
int32_t check_block(const ygg_shape* s, int32_t dtype) {
    if (int32_t rc = check_shape(s, false, false)) return rc;
    if (s->kv_dtype != dtype || (s->head_dim != 64 && s->head_dim != 128)) return YGG_ERR_UNSUPPORTED;
    if (!(s->softmax_scale > 0.f) || !std::isfinite(s->softmax_scale)) return YGG_ERR_SHAPE;
    return YGG_OK;
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

template <typename Cache>
int32_t check_cache(const Cache* c) {
    if (!c || !c->k_codes || !c->v_codes || !c->k_scale || !c->v_scale || !c->k_tail || !c->v_tail) return YGG_ERR_NULL;
    if (!aligned16(c->k_codes) || !aligned16(c->v_codes) || !aligned16(c->k_tail) || !aligned16(c->v_tail)) return YGG_ERR_UNSUPPORTED;
    if (std::is_same<Cache, ygg_block4_cache>::value && (!aligned16(c->k_scale) || !aligned16(c->v_scale))) return YGG_ERR_UNSUPPORTED;
    return YGG_OK;
}

// Shapes of ygg_prompt_attention: n_nodes rows of q, kv_capacity rows of k and v.
int32_t check_prompt(const ygg_shape* s) {
    if (!s) return YGG_ERR_NULL;
    if (s->batch < 1 || s->batch > 65535 || s->n_q_heads < 1 || s->n_kv_heads < 1 || s->n_q_heads % s->n_kv_heads != 0 || s->n_nodes < 1 ||
        s->max_seq_len < 0 || s->kv_capacity < 1 || s->kv_capacity < s->max_seq_len) return YGG_ERR_SHAPE;
    if ((s->kv_dtype != YGG_F32 && s->kv_dtype != YGG_BF16) || (s->head_dim != 64 && s->head_dim != 128)) return YGG_ERR_UNSUPPORTED;
    if (!(s->softmax_scale > 0.f) || !std::isfinite(s->softmax_scale)) return YGG_ERR_SHAPE;
    // rows of a sequence and of the batch are counted with 31 bits
    if (s->n_nodes > (1 << 25) || s->kv_capacity > 0x7fffffffLL || s->max_seq_len > (1 << 30) || (int64_t)s->n_nodes * s->n_q_heads > 0x7fffffffLL - 65536)
        return YGG_ERR_UNSUPPORTED;
    return YGG_OK;
}

int32_t check_workspace(const void* ws, size_t have, size_t need) {
    if (need == 0) return YGG_OK;
    if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255u) != 0 || have < need) return YGG_ERR_WORKSPACE;
    return YGG_OK;
}

}  // namespace

// K/V streams -- (sequence, kv head, split) or (kv head, run) -- whose workgroups all run at once: the kernel keeps a stream's row
// tiles on one XCD, which has 32 compute units, and deals the streams out over eight.  Counting all 256 compute units instead let
// 12 heads with three row tiles have seven splits: 84 streams, eleven on some XCDs, 33 workgroups and so a second round.  us per
// call by that count -> by this one: 129 rows x 4096 tokens on 12 kv heads 27.0 -> 19.4, 257 rows x 16384 on 12 82.5 -> 52.9,
// 776 rows x 8192 on 4 42.0 -> 28.1.  (Beyond 32 row tiles one round does not hold a stream; what fills the chip is left.)
static int64_t streams_at_once(int64_t row_tiles) { return row_tiles <= 32 ? 8 * (32 / row_tiles) : 256 / row_tiles; }

// Splits of every sequence's key tiles for a workgroup shape: fill the 256 CUs once -- the tile buffers leave room for one
// workgroup per CU, and a second round of workgroups pays the start-up latency again while more splits add partial-result
// traffic -- with about three key tiles per split at least (17 tiles of 49 rows on 32 kv heads: 5 / 6 / 8 splits measured
// 16.4 / 15.7 / 16.4 us per layer).
static int64_t equal_splits(const ygg_shape& s, int row_tiles, int64_t tiles) {
    int64_t ns = streams_at_once(row_tiles) / ((int64_t)s.batch * s.n_kv_heads);
    if (ns > (tiles + 2) / 3) ns = (tiles + 2) / 3;
    return ns < 1 ? 1 : ns;   // (plan_attention keeps to 64, which the merge takes)
}
// At least this many key tiles to a workgroup of the longest sequence: a batch is cut into equal runs instead (plan_attention).
static constexpr int64_t kTilesForRuns = 8;
// At least this many tiles of one sequence to a workgroup: opposite phases (plan_attention).
static constexpr int64_t kTilesForPhases128 = 10, kTilesForPhases64 = 24;
static constexpr int64_t kTilesForPhasesInRuns128 = 20, kTilesForPhasesInRuns64 = 64;

// The padded rows decide where a workgroup streams many key tiles.  Where its share of them is short, a workgroup of fewer rows
// is the better one: it starts sooner (fewer rows of Q, fewer wavefronts to meet) and its tiles take less time, so with the
// compute units filled either way the call is done sooner although each K/V byte is fetched for fewer rows.  The estimate is a
// start and a time per tile of 64 keys for each shape, in us, fitted per head_dim on calls of 129 to 516 rows, plus the merge.  On 252
// calls per head_dim (65 to 1284 rows on 4, 8, 12, 32 and 40 kv heads over 256 to 16384 tokens) its mean error is 7 % (head_dim 64:
// 11 %); the plan's shape is 1.4 % (1.7 %) slower than the best of the five on average and at most 32 % (36 %), that of fewest padded
// rows 8.9 % (8.8 %) and 43 % (54 %).  (Fitted and counted with the kernels before the last split's share and opposite phases in
// short streams, which made the first two shapes up to 10 % faster.)  The shape of fewest padded rows stays unless another promises 4 %
// less.  Measured then, us per call with the shape of fewest padded rows -> with this rule's, 8 kv heads: 196 rows x 633 tokens 17.4 -> 12.7 (tiles of 256 rows -> 64), x 4096 20.4 -> 16.6, 176 x 2078 17.8 -> 14.7 (192 -> 64), 516 x 1024
// 17.8 -> 16.7 (192 -> 64), 392 x 4096 21.7 -> 20.9 (256 -> 128); 32 kv heads: 321 rows x 4096 48.1 -> 43.2 (128 -> 192).  At
// 16384 tokens tiles of 256 lead again (392 rows: 39.0, of 128 44.3).
static void short_run_shape(const ygg_shape& s, int R, int64_t tiles, AttnPlan& p) {
    struct Kind { int32_t waves, kshares; float start, tile; };
    static constexpr Kind kinds128[] = {{8, 1, 14.0f, 1.30f}, {6, 1, 11.5f, 1.41f}, {4, 1, 10.6f, 1.15f}, {8, 2, 11.9f, 0.87f}, {4, 2, 10.5f, 0.69f}};
    static constexpr Kind kinds64[] = {{8, 1, 13.0f, 0.95f}, {6, 1, 11.3f, 1.00f}, {4, 1, 10.6f, 0.85f}, {8, 2, 11.0f, 0.66f}, {4, 2, 9.7f, 0.50f}};
    const Kind(&kinds)[5] = s.head_dim == 128 ? kinds128 : kinds64;
    constexpr float kNo = 1e30f;
    auto estimate = [&](const Kind& k) {
        const int rows = k.waves / k.kshares * 32, row_tiles = (R + rows - 1) / rows;
        if ((int64_t)s.batch * s.n_kv_heads > streams_at_once(row_tiles)) return kNo;   // more than one round of workgroups: not fitted
        int64_t ns = equal_splits(s, row_tiles, tiles);
        if (s.batch >= 2 && tiles / ns >= kTilesForRuns) return kNo;   // a batch in equal runs
        if (s.batch >= 2 && p.kshares == 1 && k.kshares > 1) return kNo;   // stays a plan that runs can serve (pairs cannot), whatever the length bound
        if (ns > 64) ns = 64;
        const float merge = ns > 1 ? 4e-7f * (float)ns * (float)s.batch * (float)s.n_kv_heads * (float)R * (float)s.head_dim : 0.f;
        return k.start + k.tile * (float)((tiles + ns - 1) / ns) + merge;
    };
    const Kind* best = nullptr;
    float least = 0.f;
    for (const Kind& k : kinds)
        if (k.waves == p.waves && k.kshares == p.kshares) least = 0.96f * estimate(k);
    if (least > 0.9f * kNo) return;
    for (const Kind& k : kinds)
        if (estimate(k) < least) { best = &k; least = estimate(k); }
    if (best) { p.waves = best->waves; p.kshares = best->kshares; }
}

// matrix-core kernels: fp16 partial outputs with one fp32 scale per row; vector kernel: fp32 partial outputs
static size_t part_o_bytes(const ygg_shape& s, bool half, int64_t nsplit) {
    return align256((size_t)nsplit * (size_t)s.batch * (size_t)s.n_nodes * (size_t)s.n_q_heads * (size_t)s.head_dim * (half ? 2 : 4));
}
static size_t part_rec_bytes(const ygg_shape& s, int64_t nsplit) {
    return align256((size_t)nsplit * (size_t)s.batch * (size_t)s.n_nodes * (size_t)s.n_q_heads * sizeof(float3));
}

AttnPlan plan_attention(const ygg_shape& s) {
    AttnPlan p{};
    const int64_t rows = (int64_t)s.batch * s.n_nodes * s.n_q_heads;
    const int64_t T = (int64_t)s.max_seq_len + s.n_nodes;
    const int64_t tiles = (T + kKeyTile - 1) / kKeyTile;
    int64_t ns;
    const bool kv8 = s.kv_dtype == YGG_FP8_E4M3;  // K/V as 8-bit codes, Q and O bf16 (head_dim 128 only)
    p.use_mfma = (s.kv_dtype == YGG_BF16 && (s.head_dim == 128 || s.head_dim == 64)) || (kv8 && s.head_dim == 128);
    if (p.use_mfma) {
        // query rows that share one K/V stream, and the workgroup shape that wastes the fewest of them
        const int R = s.n_nodes * (s.n_q_heads / s.n_kv_heads);
        p.rblocks = 1;
        p.kshares = 1;
        // Workgroup shapes, by rows per workgroup: 256 (8 wavefronts), 192 (6), 128 (8 wavefronts in
        // pairs that split every key tile), 64 and 32 (4 and 2 wavefronts in pairs).  More rows per
        // workgroup amortise the K/V tile traffic and the per-tile barrier over more matrix work, so
        // a smaller shape is taken only when it saves a good share of padded rows.
        auto padded = [R](int rw) { return (R + rw - 1) / rw * rw; };
        if (R <= 32) { p.waves = 2; p.kshares = 2; }
        else if (R <= 64) { p.waves = 4; p.kshares = 2; }
        else if (kv8) { p.waves = 4; }  // 8-bit K/V: at most four computing wavefronts, the loaders take the other slots
        else if (R <= 128) { p.waves = 8; p.kshares = 2; }
        else {
            p.waves = 8;
            int best = padded(256);
            if (padded(128) * 100 <= best * 85) { best = padded(128); p.kshares = 2; }
            // 192 rows: two of the four SIMDs carry one wavefront only, so against 256-row workgroups it has to save a
            // fifth of the rows (1284 rows x 32768 keys with 1344 instead of 1536 padded rows: 210 vs 202 us); against the
            // paired 128-row shape, which meets a barrier every 16 matrix instructions, a tenth is enough (516 rows x 4096
            // keys with 576 instead of 640 padded rows and 10 instead of 6 key splits: 27.5 vs 28.1 us per call)
            if (padded(192) * 100 <= best * (p.kshares == 2 ? 92 : 80)) { p.waves = 6; p.kshares = 1; }
        }
        if (!kv8 && R > 64) short_run_shape(s, R, tiles, p);
        int64_t ns_forced = 0;
        if (const uint64_t ov = g_plan_override.load(std::memory_order_relaxed)) {
            const int w = (int)(ov >> 56), r = (int)(ov >> 48) & 0xff, k = (int)(ov >> 40) & 0xff;
            const bool known = r == 1 && (kv8 ? (w == 4 && (k == 1 || k == 2)) || (w == 2 && k == 2)
                                              : k == 2 ? (w == 2 || w == 4 || w == 8) : (k == 1 && (w == 4 || w == 6 || w == 8)));
            if (known) { p.waves = w; p.rblocks = r; p.kshares = k; }
            ns_forced = (int64_t)(ov & 0xffffffffu);
        }
        // the widest trees (more than 900 nodes, one query head per kv head) leave no room for their masks beside 256 rows
        const int G = s.n_q_heads / s.n_kv_heads;
        while (p.kshares == 1 && p.waves > 4 && attn_mfma_smem(p.waves, 1, s.head_dim, G, s.n_nodes) > kAttnMfmaMaxSmem) p.waves -= 2;
        const int rw = p.waves / p.kshares * p.rblocks * 32;
        p.row_tiles = (R + rw - 1) / rw;
        ns = equal_splits(s, p.row_tiles, tiles);
        if (ns_forced) ns = ns_forced < tiles ? ns_forced : tiles;
        // Batches: sequence lengths live on the device and may be ragged, so instead of giving every sequence the same
        // number of splits the key tiles of all sequences are laid end to end and cut into equal runs, one per workgroup
        // of a (kv head, row tile): 256 workgroups in all, each with the same number of tiles whatever the lengths.  A
        // workgroup whose run spans two sequences starts its pipeline twice, about as long as three tiles take; where the
        // longest sequence leaves a workgroup fewer than eight tiles anyway, that costs more than the raggedness (3
        // sequences of up to 1531 tokens, 8 kv heads x 36 nodes: 21 us per call in runs, 16 in splits).
        const int64_t streams = (int64_t)s.n_kv_heads * p.row_tiles;
        const int64_t per_wg = ns > 0 ? tiles / ns : tiles;
        if (p.kshares == 1 && s.batch >= 2 && s.batch <= 256 && streams <= 128 && !ns_forced && per_wg >= kTilesForRuns) {
            int64_t slots = streams_at_once(p.row_tiles) / s.n_kv_heads;
            const int64_t most = (int64_t)s.batch * tiles;   // never more runs than tiles
            if (slots > most) slots = most;
            if (slots > 64) slots = 64;                      // the merge takes at most 64 splits per row
            if (slots >= 2) p.slots = (int32_t)slots;
        }
        // Opposite phases of the two wavefronts of a SIMD pay where a workgroup streams many tiles of one sequence: the first tile and
        // the last four go through a body with conditions, and a tile takes four barriers instead of one.  One sequence on 8 kv heads,
        // us per call without -> with them, by tiles to a workgroup, both with shares after tree_cost: 256 rows, head_dim 128, 7 tiles
        // (516 rows x 4096 tokens) 23.5 -> 23.2, 9 (1284 x 2600) 29.7 -> 30.1, 11 33.4 -> 32.3, 13 38.8 -> 36.9 and (516 x 8192) 34.8 ->
        // 32.8; head_dim 64, 13 tiles 27.4 -> 26.9, 16 (392 rows) 26.9 -> 27.4, 26 40.7 -> 39.4, 52 68.5 -> 65.9; 192 rows, head_dim 128, 4
        // tiles (516 x 2000) 19.2 -> 20.0, 7 23.1 -> 23.0, 9 (161 x 4096 on 32 kv heads) 29.9 -> 30.0, 11 (129 x 4096 on 40) 31.7 -> 29.9, 13
        // 33.0 -> 31.3.  Runs start a pipeline for every sequence they touch, their shares are not shorter for the tree's keys, and the
        // lengths may lie far below the bound that the tiles are counted from, so their line lies higher.  us per call without -> with
        // them, by tiles of the bound to a run: head_dim 128, 12 (24 sequences of 63 tokens, 208 rows on 40 kv heads) 93.5 -> 98.8, (23 of
        // 84, 776 rows on 8) 53.8 -> 56.6, 14 (7 of 203 to 407, 788 rows on 8) 35.7 -> 37.8, 10 (2 of 3000, 1284 rows on 8) 54.8 -> 55.4, 15
        // (3 of 5000, 392 rows on 8) 42.0 -> 40.6; head_dim 64, 27 (4 of 6000, 388 rows on 8) 39.8 -> 41.2, 33 (of 8192) 47.3 -> 48.2, 39 (2
        // of 6000, 1284 rows) 58.7 -> 61.4, 36 (8 of 2048, 804 rows) 51.1 -> 52.8.
        const int64_t segment = p.slots > 0 ? std::min(s.batch * tiles / p.slots, tiles) : tiles / std::clamp(ns, (int64_t)1, (int64_t)64);
        const int64_t phases_from = p.slots > 0 ? (s.head_dim == 128 ? kTilesForPhasesInRuns128 : kTilesForPhasesInRuns64)
                                                : (s.head_dim == 128 ? kTilesForPhases128 : kTilesForPhases64);
        p.phases = p.kshares == 1 && segment >= phases_from &&
                   (p.waves == 8 || (p.waves == 6 && s.head_dim == 128 && p.slots == 0));
        // What the tree's keys and their masks cost the workgroup of a sequence's last split beside their tiles, in tiles: the masks'
        // chain, and per tile of tree keys the masking, which with opposite phases lengthens both wavefronts' phases.  Such a workgroup
        // with an equal share ended 5.9 us after the others (1284 rows x 2048 tokens), 7.5 at 8192.  us per call with equal shares ->
        // these: 1284 rows x 4096 tokens on 8 kv heads 42.1 -> 36.5, x 8192 59.8 -> 55.0, x 32768 178 -> 174, 516 rows x 4096 in
        // tiles of 256 26.0 -> 24.2, 392 x 16384 41.1 -> 40.6; without opposite phases 1284 x 2048 27.6 -> 27.1.  8-bit K/V: 1284 x 4096
        // 49.6 -> 48.3, 516 x 4096 23.7 either way; where the shares stay the same the arithmetic for them shows, 140 rows x 522 on 4
        // 10.85 -> 10.95.
        const int32_t tree_tiles = (s.n_nodes + kKeyTile - 1) / kKeyTile;
        p.tree_cost = p.phases ? 1 + 6 * tree_tiles / 5 : 1 + tree_tiles / 4;
    } else {
        // vector path: one wavefront per (row, split); aim for ~4096 wavefronts
        ns = (4096 + rows - 1) / rows;
        if (ns > tiles) ns = tiles;
    }
    if (ns < 1) ns = 1;
    if (ns > 64) ns = 64;
    if (!p.use_mfma) {
        // vector kernel: equal chunks rounded up to whole key tiles; drop the splits that rounding leaves empty
        // (the matrix-core kernel deals whole tiles out evenly instead, and no split of at most `tiles` is empty)
        const int64_t chunk = ((T + ns - 1) / ns + kKeyTile - 1) / kKeyTile * kKeyTile;
        ns = (T + chunk - 1) / chunk;
    }
    p.nsplit = p.slots > 0 ? p.slots : (int32_t)ns;   // balanced batches: a sequence may span every run
    p.part_o_bytes = part_o_bytes(s, p.use_mfma, p.nsplit);
    p.part_rec_bytes = part_rec_bytes(s, p.nsplit);
    p.seq_splits_bytes = p.slots > 0 ? align256((size_t)s.batch * sizeof(int32_t)) : 0;
    return p;
}

// Workspace for this shape and every smaller max_seq_len.  More keys mean no fewer splits or runs for one workgroup shape, but
// short_run_shape changes the shape with the length, and a shorter call may take one that allows more splits: the bound is the
// workgroup shape with the most.
static size_t attention_scratch_bytes(const ygg_shape& s) {
    const AttnPlan p = plan_attention(s);
    const int R = s.n_nodes * (s.n_q_heads / s.n_kv_heads);
    int64_t most = p.nsplit;
    if (p.use_mfma && s.kv_dtype != YGG_FP8_E4M3 && R > 64) {
        const int64_t tiles = ((int64_t)s.max_seq_len + s.n_nodes + kKeyTile - 1) / kKeyTile;
        for (int rows : {256, 192, 128, 64}) most = std::max(most, std::min(equal_splits(s, (R + rows - 1) / rows, tiles), (int64_t)64));
    }
    return part_o_bytes(s, p.use_mfma, most) + part_rec_bytes(s, most) + p.seq_splits_bytes;
}

// Workgroup shapes and runs of the attention over the block cache.
BlockPlan plan_block(const ygg_shape& s, int bits) {
    BlockPlan p{};
    const int64_t R = (int64_t)s.n_nodes * (s.n_q_heads / s.n_kv_heads), row_blocks = (R + 31) / 32;
    // As many row blocks to a stream of keys as registers hold: for the 1284 rows of 321 nodes behind 32768 tokens eight take 165 us and
    // four 171.
    p.row_blocks = row_blocks <= 1 ? 1 : row_blocks <= 2 ? 2 : row_blocks <= 4 ? 4 : 8;
    p.row_tiles = (int32_t)((row_blocks + p.row_blocks - 1) / p.row_blocks);
    // One to four row blocks beyond whole tiles of eight: a smaller shape, whose wavefronts deal out the tiles of keys instead of idling
    // (those 1284 rows are five tiles and one row block: 166 us, as six tiles 212).
    if (row_blocks > 8 && row_blocks % 8 >= 1 && row_blocks % 8 <= 4) {
        p.row_tiles = (int32_t)(row_blocks / 8);
        p.rem_blocks = row_blocks % 8 <= 2 ? 2 : 4;
    }
    const int64_t per_cu = p.row_blocks == 8 ? 1 : 2;   // workgroups that a compute unit holds at once
    p.lead = p.row_blocks == 8 ? 2 : p.row_blocks == 4 ? 3 : p.row_blocks == 2 ? 4 : 6;
    // A 4-bit block takes half the time or less, a segment's own costs as long: us per call with the 8-bit cache's leads -> these, one token for
    // 16 requests of 512 to 8192 tokens 31.4 -> 28.5, 49 nodes behind 8 x 16384 tokens 123.9 -> 119.
    if (bits == 4) p.lead = p.row_blocks == 8 ? 4 : p.row_blocks == 4 ? 3 : p.row_blocks == 2 ? 8 : 15;
    p.own = 2 + (s.n_nodes + 31) / 32;
    const int64_t longest = s.max_seq_len / YGG_KV_BLOCK + p.own;      // units of a sequence
    const int64_t units = (int64_t)s.batch * (longest + p.lead);
    const int64_t most = std::min((int64_t)64, units), Hkv = s.n_kv_heads;
    // Runs: as many as fill the chip with whole rounds of workgroups, and of one to four rounds those that take least time, a round being
    // the units of a run and a start.  Workgroups beyond the whole tiles share the first round's compute units: they take rem_blocks / 8
    // of a run's time per unit.
    const int64_t slots = 256 * per_cu;
    int64_t best = 0;
    for (int64_t rounds = 1; rounds <= 4; ++rounds) {
        const int64_t at_once = slots * rounds / Hkv;      // workgroups to a kv head, over the rounds
        int64_t rem = 0, runs = 0;
        if (p.rem_blocks) {
            const int64_t all = (int64_t)p.row_blocks * p.row_tiles + p.rem_blocks;
            rem = std::clamp((at_once * p.rem_blocks + all - 1) / all, (int64_t)1, most);
            runs = std::clamp((at_once - rem) / p.row_tiles, (int64_t)1, most);
        } else {
            runs = std::clamp(rounds * per_cu * std::max(streams_at_once(p.row_tiles), (int64_t)1) / Hkv, (int64_t)1, most);
        }
        const int64_t need = ((runs * p.row_tiles + rem) * Hkv + slots - 1) / slots;
        const int64_t time = need * ((units + runs - 1) / runs + 4);
        if (rounds == 1 || time < best) { best = time; p.runs = (int32_t)runs; p.rem_runs = (int32_t)rem; }
        p.most_runs = (int32_t)std::max({runs, rem, (int64_t)p.most_runs});
    }
    // A workgroup to each sequence where that ends sooner than runs and their merge (4.5 us).  Units take 0.5, 0.6, 1.0 and 1.8 us for one,
    // two, four and eight row blocks where a workgroup has its compute unit to itself, and a little over half of that at head_dim 64.  Runs
    // are priced by the same units, without the second workgroup of a compute unit and without memory, so too low where these count: 9, 24
    // and 28 us for 3 x 2047 tokens of 65 nodes (measured 17.5), one token of 16 requests (35), 49 nodes of 8 x 4096 on 32 kv heads (64).
    // The second clause makes up for that where all sequences at their bound take memory longer than the longest takes its workgroup, for
    // bounds up to somewhere between 4096 and 8192 tokens (of 700 to 8192 the longest ends at 89 us and runs at 74).  Lengths are on the
    // device, and the even batch is the one that gains: runs -> a workgroup to each, 49 nodes, 8 sequences on 32 kv heads of 4096 tokens
    // each 64 -> 60 us, from 512 to 4096 47 -> 48, one of 4096 among seven of 128 31 -> 44.  A program whose bound is far above most
    // lengths does better with a bound beyond these.
    const float unit = (p.row_blocks == 1 ? 0.5f : p.row_blocks == 2 ? 0.6f : p.row_blocks == 4 ? 1.0f : 1.8f) * (s.head_dim == 64 ? 0.6f : 1.f);
    const int64_t groups = (int64_t)s.batch * Hkv * (p.row_tiles + (p.rem_blocks ? 1 : 0));
    const int64_t rounds = (groups + slots - 1) / slots;
    const float whole = unit * (float)(rounds * (longest + 4));
    const float stream = 2.f * (float)s.batch * (float)s.max_seq_len * (float)Hkv * (float)s.head_dim / 5.2e6f;   // us
    // Units of the 4-bit cache are short enough for that second workgroup to show: runs -> a workgroup to each, one token behind 16 x 1024 tokens
    // 18.0 -> 15.4 us, 13 nodes behind 4 x 2048 on 40 kv heads 25.6 -> 20.4, 17 behind 3 x 1024 on 12 of 64 11.8 -> 10.6; the runs that stay:
    // one token behind 2048 12.4 (16.1 in one workgroup), behind 16 x 8192 38.8 (43.0), 17 nodes behind 8 x 2048 26.8 (35.0).
    const bool shared = bits == 4 && per_cu == 2 && (int64_t)p.runs * p.row_tiles * Hkv > 256;
    if (whole < unit * (float)best * (shared ? 1.5f : 1.f) + 4.5f || (groups <= 256 && longest <= 72 && whole < stream)) {
        p.runs = p.rem_runs = 0;
        // with a compute unit to itself a workgroup takes twice the wavefronts, unless there is little to deal out to them (one token and 367
        // tokens for 16 requests 14.2 -> 11.9 us, five nodes behind 5 x 627 18.1 -> 14.9; 61 behind 3 x 139 would go 14.6 -> 16.6)
        p.wide = groups <= 256 && p.row_blocks < 8 && s.max_seq_len / YGG_KV_BLOCK >= 4;
    }
    const int32_t nsplit = std::max({p.runs, p.rem_runs, 1});
    // few rows: a whole wavefront to each in the merge
    p.merge_lanes = nsplit == 1 ? 0 : (int64_t)s.batch * s.n_nodes * s.n_q_heads <= 4096 ? 64 : s.head_dim / 8;
    p.part_o_bytes = part_o_bytes(s, true, nsplit);
    p.part_rec_bytes = part_rec_bytes(s, nsplit);
    p.seq_splits_bytes = align256(2 * (size_t)s.batch * sizeof(int32_t));
    return p;
}

// Workspace for this shape and every smaller max_seq_len: the most runs that any of them takes.
static size_t block_scratch_bytes(const ygg_shape& s, const BlockPlan& p) {
    return part_o_bytes(s, true, p.most_runs) + part_rec_bytes(s, p.most_runs) + p.seq_splits_bytes;
}

static size_t prompt_part_o_bytes(const ygg_shape& s, int64_t splits) { return align256((size_t)splits * s.n_nodes * s.n_q_heads * s.head_dim * 2); }
static size_t prompt_part_rec_bytes(const ygg_shape& s, int64_t splits) { return align256((size_t)splits * s.n_nodes * s.n_q_heads * sizeof(float3)); }

// Workgroups and key splits of the attention of prompts: row tiles of 256 or of 128 rows, and where these leave compute units without work
// their keys in parts.  The kind of least estimated time, from a start and a time per tile of 64 keys (us, fitted): 256 rows take as long per
// tile as 128 where either has its compute unit to itself, but start later, and two (head_dim 64: three) workgroups of 128 rows share one.
// us per call, 128 rows / 256: a prompt of 512 tokens with heads 32/8 of 128 15 / 21, of 2048 52 / 55, of 4096 149 / 137, of 8192 513 / 474, eight
// of 300 23 / 24, 64 of 60 24 / 29, 300 tokens behind 16000 97 / 84, 64 behind 8000 24 / 28; heads 12 of 64, 2048 tokens 24 / 32, eight of 2000
// 70 / 90, 700 behind 3000 27 / 25; 32/8 of 64, 4096 tokens 85 / 96.
// Without parts: 64 tokens behind 8000 185, 16 behind 30000 (heads 64/8) 680 (with: 23 and 35).
struct PromptKind {
    int32_t waves;
    float start, tile, shared;   // shared: time per tile of a workgroup among several
    int64_t at_once;             // workgroups on the chip
};
static const PromptKind* prompt_kinds(int head_dim) {
    static constexpr PromptKind of128[] = {{4, 6.f, 1.25f, 1.02f, 512}, {8, 14.f, 1.25f, 1.25f, 256}};
    static constexpr PromptKind of64[] = {{4, 5.f, 0.85f, 0.6f, 768}, {8, 11.f, 1.15f, 1.15f, 256}};
    return head_dim == 128 ? of128 : of64;
}
static int64_t most_prompt_splits(const PromptKind& k, int64_t groups, int64_t tiles) {
    return std::clamp(std::min(k.at_once / groups, tiles / 4), (int64_t)1, (int64_t)32);
}

PromptPlan plan_prompt(const ygg_shape& s) {
    PromptPlan p{};
    const int64_t G = s.n_q_heads / s.n_kv_heads, rows = s.n_nodes * G, Hkv = s.n_kv_heads;
    const bool f32 = s.kv_dtype == YGG_F32;
    const int64_t each = (rows + s.batch - 1) / s.batch;   // rows of a sequence, if all are alike
    const int64_t tiles = std::max((s.max_seq_len + kKeyTile - 1) / kKeyTile, 1);
    // keys of a row tile on average: half of them in a prompt from its start on, nearly all of them in one's later chunk
    const int64_t queries = (s.n_nodes + s.batch - 1) / s.batch;
    const float mean = s.max_seq_len <= 2 * queries ? 0.5f * (float)(tiles + 1) : (float)tiles - 0.5f * (float)queries / kKeyTile;
    float least = 0.f;
    for (int kind = 0; kind < 2; ++kind) {
        const PromptKind& k = prompt_kinds(s.head_dim)[kind];
        const int64_t tile = 32 * k.waves, groups = (each + tile - 1) / tile * std::min((int64_t)s.batch, rows) * Hkv;
        const int64_t most = f32 ? 1 : most_prompt_splits(k, groups, tiles);
        // parts: a merge, and partial rows written and read (512 tokens with heads 32/8 of 128 in two 17 us, in one 15)
        for (int64_t splits = most;; splits = splits / 2) {
            const int64_t all = groups * splits;
            const float share = all <= k.at_once ? (float)((all + 255) / 256) : (float)all / 256.f;   // workgroups that a compute unit gets
            const float mb = 2e-6f * (float)(splits * rows * Hkv * s.head_dim);
            const float time = k.start * (float)((all + k.at_once - 1) / k.at_once) +
                               std::max(k.tile * (float)((tiles + splits - 1) / splits), k.shared * mean / (float)splits * share) +
                               (splits > 1 ? 4.f + 0.1f * (float)splits + 0.4f * mb : 0.f);
            if (p.waves == 0 || (time < least && !f32)) {
                least = time;
                p.waves = k.waves;
                p.splits = (int32_t)splits;
            }
            if (splits == 1) break;
        }
    }
    const int64_t tile = 32 * p.waves;
    p.ranks = (int32_t)std::min(rows / tile + s.batch, rows);   // sum of ceil(rows_b / tile) over sequences that share no rows
    p.most_tiles = (int32_t)((rows + tile - 1) / tile);
    const int64_t merge = 256 / (s.head_dim / 8);
    p.merge_ranks = (int32_t)std::min(rows / merge + s.batch, rows);
    p.merge_most_tiles = (int32_t)((rows + merge - 1) / merge);
    if (p.splits > 1) {
        p.part_o_bytes = prompt_part_o_bytes(s, p.splits);
        p.part_rec_bytes = prompt_part_rec_bytes(s, p.splits);
    }
    return p;
}

// Workspace for this shape and every smaller max_seq_len: a shorter bound may take the other kind of row tiles, with as many splits as
// compute units leave it.
static size_t prompt_scratch_bytes(const ygg_shape& s) {
    if (s.kv_dtype == YGG_F32) return 0;
    const int64_t G = s.n_q_heads / s.n_kv_heads, rows = s.n_nodes * G, each = (rows + s.batch - 1) / s.batch;
    const int64_t tiles = (s.max_seq_len + kKeyTile - 1) / kKeyTile;
    int64_t most = 1;
    for (int kind = 0; kind < 2; ++kind) {
        const PromptKind& k = prompt_kinds(s.head_dim)[kind];
        const int64_t tile = 32 * k.waves, groups = (each + tile - 1) / tile * std::min((int64_t)s.batch, rows) * s.n_kv_heads;
        most = std::max(most, most_prompt_splits(k, groups, tiles));
    }
    return most > 1 ? prompt_part_o_bytes(s, most) + prompt_part_rec_bytes(s, most) : 0;
}

// Raises the shared-memory limits of the current device's kernels once; later calls cost one atomic load.
int32_t ensure_device_ready() {
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return YGG_ERR_LAUNCH;
    if (g_device_ready[dev].load(std::memory_order_acquire)) return YGG_OK;
    std::lock_guard<std::mutex> lock(g_init_mutex);
    if (g_device_ready[dev].load(std::memory_order_relaxed)) return YGG_OK;
    if (raise_limits_attn_mfma() != hipSuccess || raise_limits_expand() != hipSuccess || raise_limits_attn_block8() != hipSuccess ||
        raise_limits_attn_block4() != hipSuccess || raise_limits_attn_prompt() != hipSuccess)
        return YGG_ERR_LAUNCH;
    void* sp = nullptr;
    if (hipGetSymbolAddress(&sp, HIP_SYMBOL(scratch)) != hipSuccess || !sp) return YGG_ERR_LAUNCH;
    g_scratch_ptr[dev] = static_cast<unsigned char*>(sp);
    g_device_ready[dev].store(true, std::memory_order_release);
    return YGG_OK;
}

}  // namespace ygg

using namespace ygg;

template <typename Cache>
static int32_t attention_block_impl(const ygg_shape* s, int bits, const void* q, const Cache* cache, const int32_t* seq_lens,
                                  const void* k_tree, const void* v_tree, const int32_t* parent_idx, void* out, float* lse,
                                  void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (int32_t rc = check_block(s, bits == 8 ? YGG_FP8_BLOCK : YGG_FP4_BLOCK)) return rc;
    if (int32_t rc = check_cache(cache)) return rc;
    if (!q || !seq_lens || !k_tree || !v_tree || !parent_idx || !out) return YGG_ERR_NULL;
    if (!aligned16(q) || !aligned16(k_tree) || !aligned16(v_tree) || !aligned16(out)) return YGG_ERR_UNSUPPORTED;
    const int64_t rows = (int64_t)s->batch * s->n_nodes * s->n_q_heads;
    const BlockPlan p = plan_block(*s, bits);
    // the kernels count query rows and a batch's blocks with 31 bits, and a launch's threads with 32
    const int64_t streams = (p.runs ? (int64_t)p.runs + p.rem_runs : (int64_t)s->batch) * s->n_kv_heads + 8;
    if (rows > 0x7fffffffLL || streams * (p.row_tiles + 1) > (1 << 22) || (int64_t)s->n_nodes * s->n_q_heads > (1 << 25) ||
        (int64_t)s->batch * (s->max_seq_len / YGG_KV_BLOCK + p.lead + p.own) > 0x3fffffffLL) return YGG_ERR_UNSUPPORTED;
    if (int32_t rc = check_workspace(workspace, workspace_bytes, block_scratch_bytes(*s, p))) return rc;
    if (int32_t rc = ensure_device_ready()) return rc;

    BlockArgs a{};
    a.q = q; a.k_codes = cache->k_codes; a.v_codes = cache->v_codes; a.k_scale = cache->k_scale; a.v_scale = cache->v_scale;
    a.k_tail = cache->k_tail; a.v_tail = cache->v_tail; a.k_tree = k_tree; a.v_tree = v_tree;
    a.seq_lens = seq_lens; a.parent_idx = parent_idx;
    a.part_o = workspace;
    a.part_rec = reinterpret_cast<float3*>(static_cast<char*>(workspace) + p.part_o_bytes);
    a.seq_splits = reinterpret_cast<int32_t*>(static_cast<char*>(workspace) + p.part_o_bytes + p.part_rec_bytes);
    a.nblk = (s->kv_capacity + YGG_KV_BLOCK - 1) / YGG_KV_BLOCK;
    a.rows_total = rows;
    a.B = s->batch; a.N = s->n_nodes; a.Hq = s->n_q_heads; a.Hkv = s->n_kv_heads; a.G = a.Hq / a.Hkv; a.R = a.N * a.G;
    a.out = out; a.lse = lse;
    a.row_tiles = p.row_tiles; a.runs = p.runs; a.rem_runs = p.rem_runs; a.lead = p.lead; a.own = p.own;
    a.main_rows = p.row_tiles * p.row_blocks * 32; a.max_seq_len = s->max_seq_len; a.scale = s->softmax_scale;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const hipError_t e = bits == 8 ? launch_attn_block8(a, p, s->head_dim, st) : launch_attn_block4(a, p, s->head_dim, st);
    return e == hipSuccess ? YGG_OK : YGG_ERR_LAUNCH;
}

template <typename Cache>
static int32_t block_append_impl(const ygg_shape* s, int bits, int32_t n_layers, const void* k_new, const void* v_new, int32_t n_rows,
                          const int32_t* rows, int32_t max_new, const int32_t* n_new, const int32_t* seq_lens,
                          const Cache* cache, void* hip_stream) {
    if (int32_t rc = check_block(s, bits == 8 ? YGG_FP8_BLOCK : YGG_FP4_BLOCK)) return rc;
    if (int32_t rc = check_cache(cache)) return rc;
    if (!k_new || !v_new || !n_new || !seq_lens) return YGG_ERR_NULL;
    if (n_layers < 1 || n_layers > 65535 || n_rows < 1 || max_new < 1 || (!rows && max_new > n_rows)) return YGG_ERR_SHAPE;
    if (!aligned16(k_new) || !aligned16(v_new)) return YGG_ERR_UNSUPPORTED;
    AppendArgs a{};
    a.k_new = k_new; a.v_new = v_new; a.rows = rows; a.n_new = n_new; a.seq_lens = seq_lens;
    a.k_codes = cache->k_codes; a.v_codes = cache->v_codes; a.k_scale = cache->k_scale; a.v_scale = cache->v_scale;
    a.k_tail = cache->k_tail; a.v_tail = cache->v_tail;
    a.nblk = (s->kv_capacity + YGG_KV_BLOCK - 1) / YGG_KV_BLOCK; a.cap = s->kv_capacity;
    a.n_layers = n_layers; a.B = s->batch; a.Hkv = s->n_kv_heads; a.n_rows = n_rows; a.max_new = max_new;
    a.blocks = (int32_t)(((int64_t)max_new + YGG_KV_BLOCK - 1) / YGG_KV_BLOCK);
    if ((int64_t)n_layers * a.B * a.Hkv > (1 << 23) / a.blocks) return YGG_ERR_UNSUPPORTED;   // (the launch grid)
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const hipError_t e = bits == 8 ? launch_block8_append(a, s->head_dim, st) : launch_block4_append(a, s->head_dim, st);
    return e == hipSuccess ? YGG_OK : YGG_ERR_LAUNCH;
}

static int32_t rotary_impl(const ygg_shape* s, const void* q, int64_t q_stride, const void* k, int64_t k_stride, void* q_out, void* k_out,
                        const double* frequencies, int32_t rotary_dim, int32_t interleaved, float scale, const int32_t* seq_lens,
                        const int32_t* parent_idx, const int32_t* positions, void* hip_stream, bool norm = false,
                           const float* q_weight = nullptr, const float* k_weight = nullptr, bool per_head = false, float eps = 0.f) {
    if (!s) return YGG_ERR_NULL;
    if (!common_shape_ok(*s)) return YGG_ERR_SHAPE;
    if (!positions && s->n_nodes > kMaxNodes) return YGG_ERR_UNSUPPORTED;
    if (((s->kv_dtype < YGG_F32 || s->kv_dtype > YGG_FP8_BLOCK) && s->kv_dtype != YGG_FP4_BLOCK) || (s->head_dim != 64 && s->head_dim != 128)) return YGG_ERR_UNSUPPORTED;
    if ((!q && !k) || (q && !q_out) || (k && !k_out) || !frequencies || (!positions && (!seq_lens || !parent_idx)) ||
        (norm && ((q && !q_weight) || (k && !k_weight)))) return YGG_ERR_NULL;
    if (rotary_dim < 16 || rotary_dim > s->head_dim || !std::isfinite(scale) || !(eps >= 0.f) || !std::isfinite(eps)) return YGG_ERR_SHAPE;
    if (rotary_dim % 16) return YGG_ERR_UNSUPPORTED;
    const bool f32 = s->kv_dtype == YGG_F32;
    const int64_t q_dense = (int64_t)s->n_q_heads * s->head_dim, k_dense = (int64_t)s->n_kv_heads * s->head_dim;
    const int64_t per16 = f32 ? 4 : 8;   // elements of 16 bytes
    if (!q_stride) q_stride = q_dense;
    if (!k_stride) k_stride = k_dense;
    if ((q && (q_stride < q_dense || (q == q_out && q_stride != q_dense))) ||
        (k && (k_stride < k_dense || (k == k_out && k_stride != k_dense)))) return YGG_ERR_SHAPE;
    if ((q && (q_stride % per16 || !aligned16(q) || !aligned16(q_out))) || (k && (k_stride % per16 || !aligned16(k) || !aligned16(k_out))))
        return YGG_ERR_UNSUPPORTED;
    if (norm && ((q && !aligned16(q_weight)) || (k && !aligned16(k_weight)))) return YGG_ERR_UNSUPPORTED;
    RotaryArgs a{};
    a.q = q; a.k = k; a.q_out = q_out; a.k_out = k_out; a.frequencies = frequencies;
    a.seq_lens = seq_lens; a.parent_idx = parent_idx; a.positions = positions;
    a.q_stride = q_stride; a.k_stride = k_stride;
    a.B = s->batch; a.N = s->n_nodes; a.Hq = q ? s->n_q_heads : 0; a.Hkv = k ? s->n_kv_heads : 0; a.Dh = s->head_dim;
    const int64_t units = ((int64_t)a.Hq + a.Hkv) * (a.Dh / 16);
    if (units > (1 << 22) || s->n_nodes > (1 << 25)) return YGG_ERR_UNSUPPORTED;   // (the launch grid)
    a.units = (int32_t)units;
    a.rotary_dim = rotary_dim; a.max_seq_len = s->max_seq_len; a.scale = scale;
    a.q_weight = q_weight; a.k_weight = k_weight; a.weights_per_head = per_head; a.eps = eps;
    return launch_rotary(a, f32, interleaved != 0, norm, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? YGG_OK : YGG_ERR_LAUNCH;
}

extern "C" {

int32_t ygg_init(void) { return ensure_device_ready(); }

int32_t ygg_debug_set_attention_plan(int32_t waves, int32_t rblocks, int32_t nsplit, int32_t kshares) {
    if (waves < 0 || waves > 255 || rblocks < 0 || rblocks > 255 || kshares < 0 || kshares > 255 || nsplit < 0) return YGG_ERR_SHAPE;
    g_plan_override.store(((uint64_t)waves << 56) | ((uint64_t)rblocks << 48) | ((uint64_t)kshares << 40) | (uint32_t)nsplit,
                          std::memory_order_relaxed);
    return YGG_OK;
}

int32_t ygg_debug_attention_plan(const ygg_shape* s, int32_t* plan) {
    if (int32_t rc = check_shape(s, true, false)) return rc;
    if (!plan) return YGG_ERR_NULL;
    const AttnPlan p = plan_attention(*s);
    plan[0] = p.use_mfma; plan[1] = p.waves; plan[2] = p.kshares; plan[3] = p.row_tiles; plan[4] = p.nsplit;
    return YGG_OK;
}

int32_t ygg_debug_attention_launch(const ygg_shape* s, int32_t* launch) {
    if (int32_t rc = check_shape(s, true, false)) return rc;
    if (!launch) return YGG_ERR_NULL;
    const AttnPlan p = plan_attention(*s);
    launch[0] = p.phases; launch[1] = p.tree_cost;
    launch[2] = p.use_mfma ? (int32_t)attn_mfma_smem(p.waves, p.kshares, s->head_dim, s->n_q_heads / s->n_kv_heads, s->n_nodes) : 0;
    return YGG_OK;
}

static int32_t block_plan_impl(const ygg_shape* s, int bits, int32_t* plan) {
    if (int32_t rc = check_block(s, bits == 8 ? YGG_FP8_BLOCK : YGG_FP4_BLOCK)) return rc;
    if (!plan) return YGG_ERR_NULL;
    const BlockPlan p = plan_block(*s, bits);
    plan[0] = p.row_blocks; plan[1] = p.row_tiles; plan[2] = p.rem_blocks; plan[3] = p.runs; plan[4] = p.rem_runs;
    plan[5] = p.wide; plan[6] = p.merge_lanes;
    return YGG_OK;
}

int32_t ygg_debug_block8_plan(const ygg_shape* s, int32_t* plan) { return block_plan_impl(s, 8, plan); }
int32_t ygg_debug_block4_plan(const ygg_shape* s, int32_t* plan) { return block_plan_impl(s, 4, plan); }

int32_t ygg_debug_prompt_plan(const ygg_shape* s, int32_t* plan) {
    if (int32_t rc = check_prompt(s)) return rc;
    if (!plan) return YGG_ERR_NULL;
    const PromptPlan p = plan_prompt(*s);
    plan[0] = 32 * p.waves; plan[1] = p.splits; plan[2] = p.ranks;
    return YGG_OK;
}

const char* ygg_status_string(int32_t status) {
    switch (status) {
        case YGG_OK: return "ok";
        case YGG_ERR_NULL: return "null pointer";
        case YGG_ERR_SHAPE: return "inconsistent shape";
        case YGG_ERR_UNSUPPORTED: return "unsupported dtype, head_dim or size";
        case YGG_ERR_WORKSPACE: return "workspace missing, misaligned or too small";
        case YGG_ERR_LAUNCH: return "kernel launch failed";
        default: return "unknown status";
    }
}

size_t ygg_workspace_bytes(const ygg_shape* s, int32_t op, int32_t n_layers) {
    (void)n_layers;
    if (!s) return 0;
    switch (op) {
        case YGG_OP_ATTENTION: {
            if (check_shape(s, true, false) != YGG_OK) return 0;
            return attention_scratch_bytes(*s);
        }
        case YGG_OP_EXPAND:
        case YGG_OP_ATTACH: {
            if (check_shape(s, false, true) != YGG_OK) return 0;
            return expand_scratch_bytes(*s);
        }
        case YGG_OP_ACCEPT: {
            if (check_shape(s, false, true) != YGG_OK) return 0;
            return accept_scratch_bytes(*s);
        }
        case YGG_OP_ATTENTION_BLOCK8: {
            if (check_block(s, YGG_FP8_BLOCK) != YGG_OK) return 0;
            return block_scratch_bytes(*s, plan_block(*s, 8));
        }
        case YGG_OP_ATTENTION_BLOCK4: {
            if (check_block(s, YGG_FP4_BLOCK) != YGG_OK) return 0;
            return block_scratch_bytes(*s, plan_block(*s, 4));
        }
        case YGG_OP_PROMPT_ATTENTION: {
            if (check_prompt(s) != YGG_OK) return 0;
            return prompt_scratch_bytes(*s);
        }
        case YGG_OP_CONSTRAIN: {
            if (check_shape(s, false, true) != YGG_OK) return 0;
            return constrain_scratch_bytes(*s);
        }
        default: return 0;
    }
}

static int32_t tree_attention_impl(const ygg_shape* s, const void* q, const void* k_cache, const void* v_cache,
                                   const int32_t* seq_lens, const void* k_tree, const void* v_tree,
                                   const float* k_scale, const float* v_scale,
                                   const int32_t* parent_idx, void* out, float* lse, void* workspace,
                                   size_t workspace_bytes, void* hip_stream, bool main_only = false) {
    if (!q || !k_tree || !v_tree || !seq_lens || !parent_idx || !out) return YGG_ERR_NULL;
    if (s->max_seq_len > 0 && (!k_cache || !v_cache)) return YGG_ERR_NULL;
    // the kernels index query rows with 31 bits and address one sequence's K/V slab with 32-bit byte offsets
    const int64_t elem = s->kv_dtype == YGG_F32 ? 4 : s->kv_dtype == YGG_BF16 ? 2 : 1;
    if ((int64_t)s->batch * s->n_nodes * s->n_q_heads > 0x7fffffffLL) return YGG_ERR_UNSUPPORTED;
    if (s->kv_capacity * s->n_kv_heads * s->head_dim * elem > 0xffffffffLL) return YGG_ERR_UNSUPPORTED;
    const AttnPlan p = plan_attention(*s);
    if (int32_t rc = check_workspace(workspace, workspace_bytes, p.part_o_bytes + p.part_rec_bytes + p.seq_splits_bytes)) return rc;
    if (int32_t rc = ensure_device_ready()) return rc;

    AttnArgs a{};
    a.q = q; a.k_cache = k_cache; a.v_cache = v_cache; a.k_tree = k_tree; a.v_tree = v_tree;
    a.seq_lens = seq_lens; a.parent_idx = parent_idx; a.k_scale = k_scale; a.v_scale = v_scale;
    a.part_o = workspace;
    a.part_rec = reinterpret_cast<float3*>(static_cast<char*>(workspace) + p.part_o_bytes);
    a.seq_splits = p.slots > 0 ? reinterpret_cast<int32_t*>(static_cast<char*>(workspace) + p.part_o_bytes + p.part_rec_bytes) : nullptr;
    a.out = out; a.lse = lse;
    a.B = s->batch; a.N = s->n_nodes; a.Hq = s->n_q_heads; a.Hkv = s->n_kv_heads;
    a.G = s->n_q_heads / s->n_kv_heads; a.Dh = s->head_dim;
    a.nsplit = p.nsplit; a.max_seq_len = s->max_seq_len; a.cap = s->kv_capacity; a.scale = s->softmax_scale;
    a.slots = p.slots;
    a.lead = kSegmentLead;
    a.tree_cost = p.tree_cost;
    a.seq_runs = p.slots > 0 && p.slots % s->batch == 0 ? p.slots / s->batch : 0;
    a.S = p.slots > 0 ? a.Hkv * p.slots : a.B * a.Hkv * p.nsplit;
    a.rows_total = a.B * a.N * a.Hq;
    a.mul_nsplit = 0xffffffffu / (uint32_t)a.nsplit;
    a.mul_last = a.nsplit > 1 ? 0xffffffffu / (uint32_t)(a.nsplit - 1) : 0;   // the last split apart
    a.mul_hkv = 0xffffffffu / (uint32_t)a.Hkv;
    a.mul_g = 0xffffffffu / (uint32_t)a.G;
    a.row_tiles = p.row_tiles > 0 ? p.row_tiles : 1;
    a.mul_rt = 0xffffffffu / (uint32_t)a.row_tiles;

    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const int out_dtype = s->kv_dtype == YGG_F32 ? YGG_F32 : YGG_BF16;  // element type of Q and O
    hipError_t e = p.use_mfma ? launch_attn_mfma(a, p, st) : launch_attn_vector(a, p, s->kv_dtype, st);
    if (e != hipSuccess) return YGG_ERR_LAUNCH;
    if (main_only) return YGG_OK;
    if (p.use_mfma && p.nsplit == 1) return YGG_OK;  // the kernel wrote the final rows itself
    e = launch_attn_combine(a, p, out_dtype, st);
    return e == hipSuccess ? YGG_OK : YGG_ERR_LAUNCH;
}

int32_t ygg_tree_attention(const ygg_shape* s, const void* q, const void* k_cache, const void* v_cache,
                           const int32_t* seq_lens, const void* k_tree, const void* v_tree,
                           const int32_t* parent_idx, void* out, float* lse, void* workspace,
                           size_t workspace_bytes, void* hip_stream) {
    if (int32_t rc = check_shape(s, true, false)) return rc;
    if (s->kv_dtype == YGG_FP8_E4M3) return YGG_ERR_UNSUPPORTED;  // codes need their scales: ygg_tree_attention_fp8kv
    return tree_attention_impl(s, q, k_cache, v_cache, seq_lens, k_tree, v_tree, nullptr, nullptr, parent_idx, out, lse,
                               workspace, workspace_bytes, hip_stream);
}

int32_t ygg_debug_tree_attention_main(const ygg_shape* s, const void* q, const void* k_cache, const void* v_cache,
                                      const int32_t* seq_lens, const void* k_tree, const void* v_tree,
                                      const int32_t* parent_idx, void* out, float* lse, void* workspace,
                                      size_t workspace_bytes, void* hip_stream) {
    if (int32_t rc = check_shape(s, true, false)) return rc;
    if (s->kv_dtype == YGG_FP8_E4M3) return YGG_ERR_UNSUPPORTED;
    return tree_attention_impl(s, q, k_cache, v_cache, seq_lens, k_tree, v_tree, nullptr, nullptr, parent_idx, out, lse,
                               workspace, workspace_bytes, hip_stream, /*main_only=*/true);
}

int32_t ygg_tree_attention_fp8kv(const ygg_shape* s, const void* q, const void* k_cache, const void* v_cache,
                                 const int32_t* seq_lens, const void* k_tree, const void* v_tree,
                                 const float* k_scale, const float* v_scale, const int32_t* parent_idx, void* out,
                                 float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (int32_t rc = check_shape(s, true, false)) return rc;
    if (s->kv_dtype != YGG_FP8_E4M3) return YGG_ERR_UNSUPPORTED;
    if (!k_scale || !v_scale) return YGG_ERR_NULL;
    return tree_attention_impl(s, q, k_cache, v_cache, seq_lens, k_tree, v_tree, k_scale, v_scale, parent_idx, out, lse,
                               workspace, workspace_bytes, hip_stream);
}

int32_t ygg_equal_growth_expand(const ygg_shape* s, int32_t d, const float* draft_logits, int32_t* parent_idx,
                                int32_t* token_ids, float* cum_logprob, void* workspace, size_t workspace_bytes,
                                void* hip_stream) {
    if (int32_t rc = check_shape(s, false, true)) return rc;
    if (!draft_logits || !parent_idx || !token_ids || !cum_logprob) return YGG_ERR_NULL;
    if (s->depth < 1 || d < 1 || d > s->depth) return YGG_ERR_SHAPE;
    if ((int64_t)s->n_nodes != 1 + (int64_t)s->depth * s->width) return YGG_ERR_SHAPE;
    const ExpandPlan p = plan_expand(*s, d);
    if ((int64_t)p.F * s->vocab < s->width) return YGG_ERR_SHAPE;
    const int64_t pages = ((int64_t)s->vocab + 4095) / 4096;
    if ((int64_t)p.F * pages > 4096) return YGG_ERR_UNSUPPORTED;  // 16 M logits per sequence and step
    if ((int64_t)p.F * s->vocab >= 0x7fffffffLL) return YGG_ERR_UNSUPPORTED;  // flat candidate index is 32 bits
    if ((int64_t)s->batch * p.F > 0x7fffffffLL) return YGG_ERR_UNSUPPORTED;
    if (int32_t rc = check_workspace(workspace, workspace_bytes, p.cand_bytes + p.stat_bytes)) return rc;
    if (int32_t rc = ensure_device_ready()) return rc;

    ExpandArgs a{};
    a.logits = draft_logits; a.parent_idx = parent_idx; a.token_ids = token_ids; a.cum_logprob = cum_logprob;
    a.cands = workspace;
    a.stats = static_cast<char*>(workspace) + p.cand_bytes;
    a.B = s->batch; a.D = s->depth; a.W = s->width; a.V = s->vocab; a.N = s->n_nodes; a.d = d;
    a.F = p.F; a.chunk = p.chunk; a.nchunk = p.nchunk;
    return launch_expand(a, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? YGG_OK : YGG_ERR_LAUNCH;
}

int32_t ygg_equal_growth_expand_static(const ygg_shape* s, int32_t d, const float* draft_logits, int32_t* parent_idx,
                                       int32_t* token_ids, float* cum_logprob, void* hip_stream) {
    const size_t need = ygg_workspace_bytes(s, YGG_OP_EXPAND, 0);
    if (need > kStaticScratchBytes) return YGG_ERR_WORKSPACE;   // shape too large for the built-in scratch (0: invalid shape, reported below)
    if (int32_t rc = ensure_device_ready()) return rc;
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices || !g_scratch_ptr[dev]) return YGG_ERR_LAUNCH;
    return ygg_equal_growth_expand(s, d, draft_logits, parent_idx, token_ids, cum_logprob, g_scratch_ptr[dev],
                                   kStaticScratchBytes, hip_stream);
}

size_t ygg_attach_pool_bytes(const ygg_shape* s) {
    if (!s || check_shape(s, false, true) != YGG_OK || s->depth < 1) return 0;
    return attach_pool_bytes(*s);
}

int32_t ygg_equal_growth_attach(const ygg_shape* s, int32_t t, const float* draft_logits, int32_t* parent_idx,
                                int32_t* token_ids, float* cum_logprob, void* pool, size_t pool_bytes,
                                void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (int32_t rc = check_shape(s, false, true)) return rc;
    if (!draft_logits || !parent_idx || !token_ids || !cum_logprob || !pool) return YGG_ERR_NULL;
    if (s->depth < 1 || t < 1 || t > s->depth) return YGG_ERR_SHAPE;
    if ((int64_t)s->n_nodes != 1 + (int64_t)s->depth * s->width) return YGG_ERR_SHAPE;
    if (s->vocab < s->width) return YGG_ERR_SHAPE;  // every row must be able to offer W tokens
    const ExpandPlan p = plan_expand(*s, t);
    if (((int64_t)s->vocab + 4095) / 4096 * s->width > 4096) return YGG_ERR_UNSUPPORTED;   // 16 M logits per sequence and step
    if ((int64_t)s->n_nodes * s->vocab > 0xffffffffLL) return YGG_ERR_UNSUPPORTED;  // node*V + token is 32 bits
    if ((int64_t)s->batch * p.F > 0x7fffffffLL) return YGG_ERR_UNSUPPORTED;
    // pool + offers are sorted in one workgroup's LDS: at most 4096 entries
    if ((int64_t)p.F * s->width + (int64_t)s->width * (s->depth - t + 1) > 4096) return YGG_ERR_UNSUPPORTED;
    if ((reinterpret_cast<uintptr_t>(pool) & 15u) != 0 || pool_bytes < attach_pool_bytes(*s)) return YGG_ERR_WORKSPACE;
    if (int32_t rc = check_workspace(workspace, workspace_bytes, p.cand_bytes + p.stat_bytes)) return rc;
    if (int32_t rc = ensure_device_ready()) return rc;

    ExpandArgs a{};
    a.logits = draft_logits; a.parent_idx = parent_idx; a.token_ids = token_ids; a.cum_logprob = cum_logprob;
    a.cands = workspace;
    a.stats = static_cast<char*>(workspace) + p.cand_bytes;
    a.pool = pool; a.pool_cap = (int32_t)attach_pool_capacity(*s);
    a.B = s->batch; a.D = s->depth; a.W = s->width; a.V = s->vocab; a.N = s->n_nodes; a.d = t;
    a.F = p.F; a.chunk = p.chunk; a.nchunk = p.nchunk;
    return launch_attach(a, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? YGG_OK : YGG_ERR_LAUNCH;
}

int32_t ygg_prune_for_verification(const ygg_shape* s, int32_t w_verify, const int32_t* parent_idx,
                                   const int32_t* token_ids, const float* cum_logprob, const float* t_verifier,
                                   float t_draft, int32_t* kept_nodes, int32_t* new_parent, int32_t* new_token,
                                   float* expected_len, int32_t* best_width, void* hip_stream) {
    if (int32_t rc = check_shape(s, false, false)) return rc;
    if (!parent_idx || !token_ids || !cum_logprob || !kept_nodes || !new_parent || !new_token) return YGG_ERR_NULL;
    if (best_width && !t_verifier) return YGG_ERR_NULL;
    if (w_verify < 1 || w_verify > s->n_nodes) return YGG_ERR_SHAPE;
    if (!(t_draft >= 0.f)) return YGG_ERR_SHAPE;
    PruneArgs a{};
    a.parent_idx = parent_idx; a.token_ids = token_ids; a.cum_logprob = cum_logprob; a.t_verifier = t_verifier;
    a.kept_nodes = kept_nodes; a.new_parent = new_parent; a.new_token = new_token;
    a.expected_len = expected_len; a.best_width = best_width; a.t_draft = t_draft;
    a.B = s->batch; a.N = s->n_nodes; a.w = w_verify;
    return launch_prune(a, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? YGG_OK : YGG_ERR_LAUNCH;
}

int32_t ygg_debug_validate(const ygg_shape* s, const int32_t* parent_idx, const int32_t* seq_lens,
                           const int32_t* token_ids, const float* logits, int32_t logit_rows, int32_t* flags,
                           void* hip_stream) {
    if (int32_t rc = check_shape(s, false, token_ids != nullptr || logits != nullptr)) return rc;
    if (!flags) return YGG_ERR_NULL;
    if (logits && logit_rows < 1) return YGG_ERR_SHAPE;
    if (s->batch > 65535) return YGG_ERR_UNSUPPORTED;
    ValidateArgs a{};
    a.parent_idx = parent_idx; a.seq_lens = seq_lens; a.token_ids = token_ids; a.logits = logits; a.flags = flags;
    a.B = s->batch; a.N = s->n_nodes; a.D = s->depth; a.V = s->vocab; a.max_seq_len = s->max_seq_len;
    a.logit_rows = logit_rows;
    return launch_validate(a, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? YGG_OK : YGG_ERR_LAUNCH;
}

int32_t ygg_accept_and_compact(const ygg_shape* s, int32_t n_layers, const float* target_logits,
                               const int32_t* target_tokens, const int32_t* parent_idx, const int32_t* token_ids,
                               const void* k_tree, const void* v_tree, void* k_cache, void* v_cache,
                               int32_t* seq_lens, int32_t* accept_len, int32_t* accept_path, int32_t* bonus_token,
                               void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (int32_t rc = check_shape(s, n_layers > 0, target_logits != nullptr)) return rc;
    if (n_layers < 0 || n_layers > 65535) return YGG_ERR_SHAPE;
    if ((target_logits == nullptr) == (target_tokens == nullptr)) return YGG_ERR_NULL;
    if (!parent_idx || !token_ids || !seq_lens || !accept_len || !accept_path || !bonus_token) return YGG_ERR_NULL;
    if (n_layers > 0 && (!k_tree || !v_tree || !k_cache || !v_cache)) return YGG_ERR_NULL;
    const AcceptPlan p = plan_accept(*s);
    if ((int64_t)s->batch * s->n_nodes > 0x7fffffffLL || p.nchunk > 65535) return YGG_ERR_UNSUPPORTED;
    if (int32_t rc = check_workspace(workspace, workspace_bytes, p.part_bytes + p.oldlen_bytes)) return rc;

    AcceptArgs a{};
    a.target_logits = target_logits; a.target_tokens = target_tokens;
    a.parent_idx = parent_idx; a.token_ids = token_ids;
    a.k_tree = k_tree; a.v_tree = v_tree; a.k_cache = k_cache; a.v_cache = v_cache;
    a.seq_lens = seq_lens; a.accept_len = accept_len; a.accept_path = accept_path; a.bonus_token = bonus_token;
    a.part = workspace;
    a.old_len = reinterpret_cast<int32_t*>(static_cast<char*>(workspace) + p.part_bytes);
    a.B = s->batch; a.N = s->n_nodes; a.D = s->depth; a.V = s->vocab; a.Hkv = s->n_kv_heads; a.Dh = s->head_dim;
    a.n_layers = n_layers; a.chunk = p.chunk; a.nchunk = p.nchunk; a.max_seq_len = s->max_seq_len;
    a.elem_bytes = s->kv_dtype == YGG_F32 ? 4 : s->kv_dtype == YGG_BF16 ? 2 : 1; a.cap = s->kv_capacity;
    return launch_accept(a, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? YGG_OK : YGG_ERR_LAUNCH;
}

int32_t ygg_tree_attention_block8(const ygg_shape* s, const void* q, const ygg_block8_cache* cache, const int32_t* seq_lens,
                                  const void* k_tree, const void* v_tree, const int32_t* parent_idx, void* out, float* lse,
                                  void* workspace, size_t workspace_bytes, void* hip_stream) {
    return attention_block_impl(s, 8, q, cache, seq_lens, k_tree, v_tree, parent_idx, out, lse, workspace, workspace_bytes, hip_stream);
}

int32_t ygg_tree_attention_block4(const ygg_shape* s, const void* q, const ygg_block4_cache* cache, const int32_t* seq_lens,
                                  const void* k_tree, const void* v_tree, const int32_t* parent_idx, void* out, float* lse,
                                  void* workspace, size_t workspace_bytes, void* hip_stream) {
    return attention_block_impl(s, 4, q, cache, seq_lens, k_tree, v_tree, parent_idx, out, lse, workspace, workspace_bytes, hip_stream);
}

int32_t ygg_block8_append(const ygg_shape* s, int32_t n_layers, const void* k_new, const void* v_new, int32_t n_rows,
                          const int32_t* rows, int32_t max_new, const int32_t* n_new, const int32_t* seq_lens,
                          const ygg_block8_cache* cache, void* hip_stream) {
    return block_append_impl(s, 8, n_layers, k_new, v_new, n_rows, rows, max_new, n_new, seq_lens, cache, hip_stream);
}

int32_t ygg_block4_append(const ygg_shape* s, int32_t n_layers, const void* k_new, const void* v_new, int32_t n_rows,
                          const int32_t* rows, int32_t max_new, const int32_t* n_new, const int32_t* seq_lens,
                          const ygg_block4_cache* cache, void* hip_stream) {
    return block_append_impl(s, 4, n_layers, k_new, v_new, n_rows, rows, max_new, n_new, seq_lens, cache, hip_stream);
}

int32_t ygg_tree_rotary(const ygg_shape* s, const void* q, int64_t q_stride, const void* k, int64_t k_stride, void* q_out, void* k_out,
                        const double* frequencies, int32_t rotary_dim, int32_t interleaved, float scale, const int32_t* seq_lens,
                        const int32_t* parent_idx, const int32_t* positions, void* hip_stream) {
    return rotary_impl(s, q, q_stride, k, k_stride, q_out, k_out, frequencies, rotary_dim, interleaved, scale, seq_lens, parent_idx, positions,
                       hip_stream);
}

int32_t ygg_tree_norm_rotary(const ygg_shape* s, const void* q, int64_t q_stride, const void* k, int64_t k_stride, void* q_out, void* k_out,
                             const float* q_weight, const float* k_weight, int32_t weights_per_head, float eps, const double* frequencies,
                             int32_t rotary_dim, int32_t interleaved, float scale, const int32_t* seq_lens, const int32_t* parent_idx,
                             const int32_t* positions, void* hip_stream) {
    return rotary_impl(s, q, q_stride, k, k_stride, q_out, k_out, frequencies, rotary_dim, interleaved, scale, seq_lens, parent_idx, positions,
                       hip_stream, true, q_weight, k_weight, weights_per_head != 0, eps);
}

int32_t ygg_prompt_attention(const ygg_shape* s, const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                             int64_t v_stride, const int32_t* q_first, const int32_t* q_len, const int32_t* k_first, const int32_t* k_len,
                             void* out, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (int32_t rc = check_prompt(s)) return rc;
    if (!q || !k || !v || !q_first || !q_len || !k_first || !k_len || !out) return YGG_ERR_NULL;
    const bool f32 = s->kv_dtype == YGG_F32;
    const int64_t q_dense = (int64_t)s->n_q_heads * s->head_dim, k_dense = (int64_t)s->n_kv_heads * s->head_dim, per16 = f32 ? 4 : 8;
    if (!q_stride) q_stride = q_dense;
    if (!k_stride) k_stride = k_dense;
    if (!v_stride) v_stride = k_dense;
    if (q_stride < q_dense || k_stride < k_dense || v_stride < k_dense) return YGG_ERR_SHAPE;
    if (q_stride % per16 || k_stride % per16 || v_stride % per16 || !aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out))
        return YGG_ERR_UNSUPPORTED;
    if (k_stride > (1 << 24) || v_stride > (1 << 24)) return YGG_ERR_UNSUPPORTED;   // (32-bit offsets inside a tile of keys)
    const PromptPlan p = plan_prompt(*s);
    if ((int64_t)p.ranks * s->n_kv_heads * p.splits > (1 << 22) || (p.splits > 1 && (int64_t)p.merge_ranks * s->n_kv_heads > (1 << 23)))
        return YGG_ERR_UNSUPPORTED;   // (the launch grid)
    if (int32_t rc = check_workspace(workspace, workspace_bytes, prompt_scratch_bytes(*s))) return rc;
    if (int32_t rc = ensure_device_ready()) return rc;
    PromptArgs a{};
    a.q = q; a.k = k; a.v = v; a.q_first = q_first; a.q_len = q_len; a.k_first = k_first; a.k_len = k_len;
    a.part_o = workspace;
    a.part_rec = reinterpret_cast<float3*>(static_cast<char*>(workspace) + p.part_o_bytes);
    a.out = out; a.lse = lse; a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride; a.k_rows = s->kv_capacity;
    a.B = s->batch; a.Hq = s->n_q_heads; a.Hkv = s->n_kv_heads; a.G = a.Hq / a.Hkv; a.q_rows = s->n_nodes; a.max_keys = s->max_seq_len;
    a.splits = p.splits; a.most_tiles = p.most_tiles; a.scale = s->softmax_scale;
    return launch_attn_prompt(a, p, s->head_dim, f32, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? YGG_OK : YGG_ERR_LAUNCH;
}

int32_t ygg_count_tokens(const ygg_shape* s, const int32_t* tokens, int32_t n_tokens, const int32_t* rows, int32_t first, int32_t max_new,
                         const int32_t* n_new, int32_t prompt, int32_t* counts, void* hip_stream) {
    if (int32_t rc = check_shape(s, false, true)) return rc;
    if (!tokens || !n_new || !counts) return YGG_ERR_NULL;
    if (n_tokens < 1 || max_new < 1 || first < 0) return YGG_ERR_SHAPE;
    CountArgs a{};
    a.tokens = tokens; a.rows = rows; a.n_new = n_new; a.counts = counts;
    a.B = s->batch; a.V = s->vocab; a.n_tokens = n_tokens; a.first = first; a.max_new = max_new; a.prompt = prompt != 0;
    return launch_count(a, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? YGG_OK : YGG_ERR_LAUNCH;
}

int32_t ygg_constrain_logits(const ygg_shape* s, const void* logits, int32_t logits_dtype, int64_t row_stride, const int32_t* parent_idx,
                             const int32_t* token_ids, const ygg_logit_rules* rules, float* out, int32_t* best, void* workspace,
                             size_t workspace_bytes, void* hip_stream) {
    if (int32_t rc = check_shape(s, false, true)) return rc;
    if (!logits || !parent_idx || !token_ids || !rules || (!out && !best)) return YGG_ERR_NULL;
    if (logits_dtype != YGG_F32 && logits_dtype != YGG_BF16) return YGG_ERR_UNSUPPORTED;
    if (!row_stride) row_stride = s->vocab;
    if (row_stride < s->vocab) return YGG_ERR_SHAPE;
    if (static_cast<const void*>(out) == logits && (logits_dtype != YGG_F32 || row_stride != s->vocab)) return YGG_ERR_SHAPE;
    if (rules->masks && !rules->mask_index) return YGG_ERR_NULL;
    if (rules->masks && rules->n_masks < 1) return YGG_ERR_SHAPE;
    const int64_t rows = (int64_t)s->batch * s->n_nodes;
    if (rows > (1 << 23) || s->vocab > (1 << 28)) return YGG_ERR_UNSUPPORTED;   // (the launch grid)
    if (best)
        if (int32_t rc = check_workspace(workspace, workspace_bytes, constrain_scratch_bytes(*s))) return rc;
    ConstrainArgs a{};
    a.logits = logits; a.parent_idx = parent_idx; a.token_ids = token_ids; a.counts = rules->counts; a.repetition = rules->repetition;
    a.presence = rules->presence; a.frequency = rules->frequency; a.bias = rules->bias; a.masks = rules->masks;
    a.mask_index = rules->mask_index; a.out = out; a.best = best; a.part = workspace; a.row_stride = row_stride;
    a.B = s->batch; a.N = s->n_nodes; a.V = s->vocab; a.bias_shared = rules->bias_shared != 0; a.n_masks = rules->n_masks;
    return launch_constrain(a, logits_dtype == YGG_F32, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? YGG_OK : YGG_ERR_LAUNCH;
}

}  // extern "C"
