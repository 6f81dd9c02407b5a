// What appending to the 8-bit and to the 4-bit block cache shares: which rows a workgroup has, and the rows that stay open.
#pragma once
#include "ygg_internal.h"
#include "ygg_device.h"

namespace ygg {
namespace block_cache {

constexpr int kT = YGG_KV_BLOCK;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;

// The largest bits of the magnitudes of eight values in either half of a word (magnitudes are in the order of their bits).
__device__ __forceinline__ u16x2 magnitude8(const u32x4 v, u16x2 m) {
#pragma unroll
    for (int e = 0; e < 4; ++e) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, v[e] & 0x7fff7fffu));
    return m;
}
__device__ __forceinline__ float largest(u16x2 m) { return __uint_as_float((uint32_t)max(m[0], m[1]) << 16); }
__device__ __forceinline__ u32x4 fetch(const uint16_t* row, int d) {   // a null row is one of zeros
    u32x4 x = {};
    if (row) x = *reinterpret_cast<const u32x4*>(row + d);
    return x;
}

// Workgroup blockIdx.x is one (layer, sequence, kv head, touched block).
struct Touched {
    int64_t old, end, t0, at;   // lengths before and after; the block's first token, and its number in the cache's arrays
    bool complete, first;       // all of the block's tokens are there now; it is the first touched one
    int64_t row;                // elements of a token
    const uint16_t *k_new, *v_new;
    uint16_t *k_tail, *v_tail;
    const int32_t* rows;
    int64_t n_rows;
    int dh;

    __device__ __forceinline__ Touched(const AppendArgs& a, int head_dim) {
        int64_t w = blockIdx.x;
        const int j = (int)(w % a.blocks); w /= a.blocks;
        const int g = (int)(w % a.Hkv); w /= a.Hkv;
        const int b = (int)(w % a.B);
        const int64_t lb = w;                 // layer * B + b
        const int64_t len = a.seq_lens[b];
        end = len < 0 ? 0 : (len > a.cap ? a.cap : len);
        const int64_t want = a.n_new[b];
        int64_t fresh = want < 0 ? 0 : (want > a.max_new ? a.max_new : want);
        if (fresh > end) fresh = end;
        old = end - fresh;
        const int64_t block = old / kT + j;
        t0 = block * kT;
        complete = t0 + kT <= end && fresh > 0;
        first = j == 0;
        dh = head_dim;
        row = (int64_t)a.Hkv * dh;
        k_new = static_cast<const uint16_t*>(a.k_new) + lb * a.n_rows * row + (int64_t)g * dh;
        v_new = static_cast<const uint16_t*>(a.v_new) + lb * a.n_rows * row + (int64_t)g * dh;
        k_tail = static_cast<uint16_t*>(a.k_tail) + lb * 2 * kT * row + (int64_t)g * dh;
        v_tail = static_cast<uint16_t*>(a.v_tail) + lb * 2 * kT * row + (int64_t)g * dh;
        rows = a.rows ? a.rows + (int64_t)b * a.max_new : nullptr;
        n_rows = a.n_rows;
        at = (lb * a.Hkv + g) * a.nblk + block;
    }
    __device__ __forceinline__ int64_t new_row(int64_t token) const {   // row of the caller's tensor, or -1
        const int64_t k = token - old;
        const int64_t r = rows ? (int64_t)rows[k] : k;
        return r >= 0 && r < n_rows ? r : -1;
    }
    // a token's row of the block, or null: zeros
    __device__ __forceinline__ const uint16_t* k_row(int64_t token) const { return row_at(token, k_tail, k_new); }
    __device__ __forceinline__ const uint16_t* v_row(int64_t token) const { return row_at(token, v_tail, v_new); }
    __device__ __forceinline__ const uint16_t* row_at(int64_t token, const uint16_t* tail, const uint16_t* fresh_rows) const {
        if (token < old) return tail + token % (2 * kT) * row;
        const int64_t r = new_row(token);
        return r >= 0 ? fresh_rows + r * row : nullptr;
    }
    // The workgroup of the first touched block copies the rows that stay open, after it has read that block's old rows.  (Those that
    // complete a block are in its codes, and nothing reads them from the tail: the header says how far back a length may be taken.)
    __device__ __forceinline__ void keep_open_rows(const AppendArgs& a, int tid) const {
        if (!first) return;
        const int64_t open = max(end / kT * kT, old);
        for (int64_t p = tid; p < (end - open) * (dh / 8); p += 256) {
            const int64_t token = open + p / (dh / 8), r = new_row(token);
            const int64_t d = p % (dh / 8) * 8;
            u32x4 k = {}, v = {};
            if (r >= 0) {
                k = *reinterpret_cast<const u32x4*>(k_new + r * row + d);
                v = *reinterpret_cast<const u32x4*>(v_new + r * row + d);
            }
            *reinterpret_cast<u32x4*>(k_tail + token % (2 * kT) * row + d) = k;
            *reinterpret_cast<u32x4*>(v_tail + token % (2 * kT) * row + d) = v;
        }
    }
};

}  // namespace block_cache
}  // namespace ygg
