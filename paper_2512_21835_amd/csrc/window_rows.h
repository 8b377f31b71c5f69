// What the window attention kernels (window.hip, window_f32.hip) share: which keys a row sees, the rows of a workgroup
// and the tiles of keys that they see, four elements of a row, numbers as sums of bf16 terms.
#pragma once

#include <hip/hip_runtime.h>

#include "lanes.h"
#include "ops_kernels.h"
#include "pair.h"
#include "stage_ops.h"

namespace stg {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef short s16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef const __attribute__((address_space(4))) int *const_ints;
typedef __attribute__((address_space(3))) u32x4 *lds16;
typedef __attribute__((address_space(3))) s16x4_t *lds8;
typedef __attribute__((address_space(3))) float *lds4;

constexpr int kPage = kBlockTokens;
constexpr long kMaxBlocks = (1L << 24) - 1;   // workgroups of 256 in a grid: their threads are counted in 32 bits
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kSlack = 8.f;
constexpr float kMaxBf16 = 0x1.FEp127f;
// Probabilities and sums of up to 2^24 keys are scaled by this where values near the largest number are added up.
constexpr int kRoomBits = 24;
constexpr float kRoom = 1.f / (1 << kRoomBits);

// The same in every lane, and known to be.
__device__ __forceinline__ OpRows::Seq uniform(OpRows::Seq s) {
    const uint64_t t = (uint64_t)(uintptr_t)s.table;
    const uint32_t low = __builtin_amdgcn_readfirstlane((uint32_t)t), high = __builtin_amdgcn_readfirstlane((uint32_t)(t >> 32));
    return {__builtin_amdgcn_readfirstlane(s.first), __builtin_amdgcn_readfirstlane(s.n), __builtin_amdgcn_readfirstlane(s.pos0),
            reinterpret_cast<const int *>((uintptr_t)((uint64_t)high << 32 | low))};
}

// Inclusive sums over the lanes (DPP: within rows of 16, then row to row).
__device__ __forceinline__ int lane_scan(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);   // row_shr 1, 2, 4, 8
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);   // row_bcast 15: rows 0, 2 to 1, 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);   // row_bcast 31: row 1 to 2 and 3
    return v;
}
__device__ __forceinline__ const int *lane_pointer(const int *p, int lane) {
    const uint64_t t = (uint64_t)(uintptr_t)p;
    const uint32_t low = __builtin_amdgcn_readlane((uint32_t)t, lane), high = __builtin_amdgcn_readlane((uint32_t)(t >> 32), lane);
    return reinterpret_cast<const int *>((uintptr_t)((uint64_t)high << 32 | low));
}

__device__ __forceinline__ bool sees(const WindowArgs &a, int pos, int key) {
    return (key <= pos) & (key < a.rows.max_len) & ((key > pos - a.window) | (key < a.sinks));   // (no branches)
}
// Whether rows at positions first .. last all see keys k0 .. k0 + n - 1.
__device__ __forceinline__ bool all_see(const WindowArgs &a, int first, int last, int k0, int n) {
    return k0 + n - 1 <= first && k0 + n <= a.rows.max_len && (k0 > last - a.window || k0 + n <= a.sinks);
}

__device__ __forceinline__ void load4(const void *p, size_t e, int type, float v[4]) {
    if (type == STAGE_F32) {
        const float4 x = *reinterpret_cast<const float4 *>(static_cast<const float *>(p) + e);
        v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
    } else {
        const uint2 x = *reinterpret_cast<const uint2 *>(static_cast<const uint16_t *>(p) + e);
        v[0] = __uint_as_float(x.x << 16); v[1] = __uint_as_float(x.x & 0xFFFF0000u);
        v[2] = __uint_as_float(x.y << 16); v[3] = __uint_as_float(x.y & 0xFFFF0000u);
    }
}
// (kPair: rows of a multiple of 32 elements, so the pair of element e of many rows is at pair_at(e))
constexpr int kPair = -1;
__device__ __forceinline__ void store4(void *p, size_t e, int type, float4 v) {
    if (type == kPair) {
        store_pair4(static_cast<uint16_t *>(p) + pair_at((long)e), v);
    } else if (type == STAGE_F32) {
        *reinterpret_cast<float4 *>(static_cast<float *>(p) + e) = v;
    } else {
        typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
        *reinterpret_cast<bf16x4 *>(static_cast<uint16_t *>(p) + e) = bf16x4{(__bf16)v.x, (__bf16)v.y, (__bf16)v.z, (__bf16)v.w};
    }
}
// o / l; a row that saw no key is 0.
__device__ __forceinline__ float4 quotient(float4 o, float l) {
    const float r = l == 0.f ? 0.f : 1.f / l;
    return make_float4(o.x * r, o.y * r, o.z * r, o.w * r);
}

// bf16 terms of a probability, by those of q: three with fp32 rows.  With bf16 rows two, which hold it to 2^-16 of its value,
// well below a step of the output; one alone leaves 2^-8 in every product, and the output as far off again as its own rounding.
constexpr int p_terms(int q_terms) { return q_terms == 1 ? 2 : q_terms; }

// x as a sum of bf16 terms, each the nearest to what the ones before leave: term 1 is at most 2^-8 of x, term 2 2^-17, and
// three hold all 24 bits.
template <int TERMS>
__device__ __forceinline__ void split_terms(float x, __bf16 t[TERMS]) {
#pragma unroll
    for (int i = 0; i < TERMS; ++i) {
        t[i] = (__bf16)x;
        x -= (float)t[i];
    }
}

// Two numbers (a in the low halves) at once.
template <int TERMS>
__device__ __forceinline__ void split_terms2(float a, float b, uint32_t t[TERMS]) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < TERMS; ++i) {
        t[i] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
        if (i == TERMS - 1) break;
        a -= __uint_as_float(t[i] << 16);
        b -= __uint_as_float(t[i] & 0xFFFF0000u);
    }
}

// Bits 0 .. n of a word.
__device__ __forceinline__ uint32_t bits_to(int n) { return n < 0 ? 0u : ~0u >> (31 - min(n, 31)); }
// sees(), for the 32 keys from k0 on.
__device__ __forceinline__ uint32_t seen_bits(const WindowArgs &a, int pos, int k0) {
    return bits_to(min(pos, a.rows.max_len - 1) - k0) & (~bits_to(pos - a.window - k0) | bits_to(a.sinks - 1 - k0));
}
// -inf for the scores i whose bit 8 (i / 4) + i % 4 is not set.
__device__ __forceinline__ void hide_scores(f32x16_t &s, uint32_t seen) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const uint32_t yes = (uint32_t)((int)(seen << (31 - 8 * (i / 4) - i % 4)) >> 31);
        s[i] = __uint_as_float((__float_as_uint(s[i]) & yes) | (0xFF800000u & ~yes));
    }
}

// Numbers t as ranges: below `low`, or of [from, from + n).  (Scalar work counts: a turn has few hundred cycles.)
struct Turns {
    int low, from;
    unsigned n;
    __device__ __forceinline__ bool has(int t) const { return (t < low) | ((unsigned)(t - from) < n); }
};

// 2^log_bq consecutive rows of a sequence (the blocks of all sequences in turn, of each its last rows first, which see
// the most keys), and the tiles of 32 keys that they see: 0 .. sink - 1, then from, from + 1, ...; n_tiles in all.
constexpr int kTileKeys = 32;
struct RowBlock {
    OpRows::Seq seq;
    int t0, rows, first;       // first row within the sequence, rows, position of the first
    int end, last_page;        // keys from `end` on are seen by no row
    int sink, from, n_tiles;

    // false: there are fewer blocks
    __device__ __forceinline__ bool find(const WindowArgs &a, int block, int log_bq) {
        const int lane = __lane_id(), bq = 1 << log_bq;
        for (int i0 = 0;; i0 += 64) {   // 64 sequences at a time
            if (i0 >= a.rows.n_seqs) return false;
            const OpRows::Seq at = a.rows.seq(min(i0 + lane, a.rows.n_seqs - 1));
            const int own = i0 + lane < a.rows.n_seqs ? (min(at.n, a.rows.max_rows) + bq - 1) >> log_bq : 0, sum = lane_scan(own);
            const int before = __popcll(__builtin_amdgcn_ballot_w64(sum <= block));   // (sums ascend)
            if (before < 64) {
                block = __builtin_amdgcn_readlane(sum, before) - 1 - block;
                seq = {__builtin_amdgcn_readlane(at.first, before), __builtin_amdgcn_readlane(at.n, before),
                       __builtin_amdgcn_readlane(at.pos0, before), lane_pointer(at.table, before)};
                break;
            }
            block -= __builtin_amdgcn_readlane(sum, 63);
        }
        t0 = block << log_bq;
        rows = min(bq, min(seq.n, a.rows.max_rows) - t0);
        first = seq.pos0 + t0;
        end = min(first + rows, a.rows.max_len);
        last_page = max(end - 1, 0) / kPage;
        sink = (max(0, min(a.sinks, end)) + kTileKeys - 1) / kTileKeys;
        from = max(max(0, first - a.window + 1) / kTileKeys, sink);
        n_tiles = end <= 0 ? 0 : sink + max(0, (end + kTileKeys - 1) / kTileKeys - from);
        return true;
    }
    // whether some row sees the key
    __device__ __forceinline__ bool sees(const WindowArgs &a, int key) const {
        return (key < end) & ((key > first - a.window) | (key < a.sinks));
    }
    __device__ __forceinline__ int tile_at(int t) const { return t < sink ? t : from + t - sink; }
    // page h of tile t, of those that hold a key of the sequence
    __device__ __forceinline__ int page_at(int t, int h) const { return min(2 * tile_at(t) + h, last_page); }
    // tiles that rows at positions r0 .. r1 (r0 <= r1) all see, and those with a key that some of them sees
    __device__ __forceinline__ Turns whole(const WindowArgs &a, int r0, int r1) const {
        Turns w;
        w.low = min(sink, max(0, min(min(a.sinks, r0 + 1), a.rows.max_len)) / kTileKeys);
        w.from = sink + max(0, max(0, r1 - a.window + kTileKeys) / kTileKeys - from);
        w.n = max(0, sink + max(0, min(r0 + 1, a.rows.max_len)) / kTileKeys - from - w.from);
        return w;
    }
    __device__ __forceinline__ Turns touched(const WindowArgs &a, int r0, int r1) const {
        Turns w;
        w.low = min(sink, (max(0, min(min(a.sinks, r1 + 1), a.rows.max_len)) + kTileKeys - 1) / kTileKeys);
        w.from = sink + max(0, max(0, r0 - a.window + 1) / kTileKeys - from);
        w.n = max(0, sink + (max(0, min(r1 + 1, a.rows.max_len)) + kTileKeys - 1) / kTileKeys - from - w.from);
        return w;
    }
};
// Numbers by size, those that are not finite from 0x7F800000 on.
__device__ __forceinline__ uint32_t size_bits(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }
// Whether the state of the lane's column holds what is not finite.
template <int NB>
__device__ __forceinline__ bool not_finite(float l, const f32x16_t (&o)[NB]) {
    uint32_t most = size_bits(l);
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) most = max(most, size_bits(o[b][i]));
    return most >= 0x7F800000u;
}

// The column of a lane (and of lane ^ 32: d 32 c + 8 j + 4 (lane / 32) + i in o[c][4 j + i]) key by key in fp32, where terms
// cannot give it: an infinity has none, and 0 x inf in the matrix instructions meets columns that do not see it.  Columns
// marked `again` (sums that pass the largest number among them: scaled by kRoom, they do not), and those that see a K or V
// that is not finite, or too large to be rounded to bf16 (looked for if some are there); others keep o and l.
template <int D, int TYPE, int KV_TYPE>
__device__ __forceinline__ void by_keys(const WindowArgs &a, const RowBlock &rb, int g, size_t q_at, int pos, bool again, bool some,
                                        f32x16_t (&o)[D / 32], float &l) {
    const int half = __lane_id() >> 5;
    const size_t head = (size_t)kPage * D;
    auto each_key = [&](bool all, auto use) {   // until !use(key, place of K, place of V), the lane's half of them
#pragma unroll 1
        for (int i = 0; all && i < rb.n_tiles * kTileKeys; ++i) {
            const int key = rb.tile_at(i / kTileKeys) * kTileKeys + i % kTileKeys;
            if (key / kPage > rb.last_page) continue;
            const int b = ((const_ints)(uintptr_t)rb.seq.table)[key / kPage];
            if ((unsigned)b >= (unsigned)a.rows.n_blocks) continue;
            const size_t k = ((size_t)b * 2 * a.n_kv_heads + g) * head + key % kPage * D;
            all = use(key, k + 8 * half, k + a.n_kv_heads * head + 4 * half);
        }
    };
    each_key(some, [&](int key, size_t k, size_t v) {
        uint32_t most = 0;
        float x[4];
#pragma unroll 1
        for (int c = 0; c < D; c += 16)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                load4(a.pool, k + c + 4 * h, KV_TYPE, x);
#pragma unroll
                for (int e = 0; e < 4; ++e) most = max(most, size_bits(x[e]));
                load4(a.pool, v + c + 8 * h, KV_TYPE, x);
#pragma unroll
                for (int e = 0; e < 4; ++e) most = max(most, size_bits(x[e]));
            }
        again |= sees(a, pos, key) & (most > size_bits(kMaxBf16));
        return true;
    });
    again = __shfl_xor((int)again, 32) | (int)again;
    float m = -INFINITY;
    bool done = !again;   // (a score that is NaN makes the column NaN, whatever follows)
    l = again ? 0.f : l;
#pragma unroll
    for (int b = 0; b < D / 32; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[b][i] = again ? 0.f : o[b][i];
    each_key(true, [&](int key, size_t k, size_t v) {
        float w = 0.f;
#pragma unroll 1
        for (int kk = 0; kk < D / 16; ++kk) {
            float x[8], y[8];
            load4(a.q, q_at + 16 * kk, TYPE, x);
            load4(a.q, q_at + 16 * kk + 4, TYPE, x + 4);
            load4(a.pool, k + 16 * kk, KV_TYPE, y);
            load4(a.pool, k + 16 * kk + 4, KV_TYPE, y + 4);
#pragma unroll
            for (int j = 0; j < 8; ++j) w = fmaf(x[j], y[j], w);
            asm volatile("" ::: "memory");   // (registers)
        }
        w = (w + lane_xor(w, 32)) * a.scale * kLog2e;
        const bool seen = again & sees(a, pos, key);
        const float to = seen & (w > m) ? w : m, ref = to == -INFINITY ? 0.f : to;
        const float alpha = again ? __builtin_amdgcn_exp2f(m - ref) : 1.f;
        w = seen ? __builtin_amdgcn_exp2f(w - ref) * kRoom : 0.f;
        m = to;
        l = l * alpha + (half ? 0.f : w);   // (the halves of a column are added up at the end)
#pragma unroll
        for (int c = 0; c < D / 32; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float x[4];
                load4(a.pool, v + 32 * c + 8 * j, KV_TYPE, x);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[c][4 * j + e] = o[c][4 * j + e] * alpha + (seen ? w * x[e] : 0.f);
                __builtin_amdgcn_sched_barrier(0);   // (registers)
            }
        done |= w != w;
        l = done & again ? NAN : l;
        return __builtin_amdgcn_ballot_w64(!done) != 0;
    });
}
// With a turn before and a turn behind each run.
__device__ __forceinline__ Turns widened(Turns w) {
    return {w.low > 0 ? w.low + 1 : 0, w.from - 1, w.n ? w.n + 2 : 0};
}

}  // namespace
}  // namespace stg
