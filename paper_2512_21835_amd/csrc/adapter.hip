// Low-rank adapters of many requests beside a shared projection: out = base + scale B (A x), a pair (A, B) per row.
//
// Two launches.  Down: t = A x over slices of k, whose sums go to the workspace; up: the slices added, out = base + scale B
// t.  Both take tiles of 16 rows as the columns of 16x16x32 MFMAs and loop over the adapters that occur in the tile; a
// product of another row's adapter is dropped with its column, so no row's values meet another's.  Bound by bytes: A
// and B of the adapters present (decode), x, base and out (prompts).  fp32 operands enter as the exact sum of three
// bf16 terms.
//
// Every operand goes through LDS, with neighbouring lanes side by side in memory (weights by copies straight into a
// ring of each wavefront's own): an MFMA operand read straight from memory has neighbouring lanes in different rows,
// 55 cache accesses per instruction, which alone took 30 of the up kernel's 53 us at 64 rows of a 70B-shaped projection.
//
// Down and up: 16 rows of 16 adapters of rank 16, 4096 x 4096, fp32, 5.6 + 6.6 us (latency of the launches); 64 bf16 rows of
// 48 adapters up to rank 64, 8192 x 28672 (135 MB), 9 + 32 us (the up kernel 4 TB/s); 4001 bf16 rows of 3 adapters of rank
// 32, 5120 x 5120 (125 MB), 16.6 + 26 us (3.2 TB/s: a block's base is copied one block ahead only).
#include <type_traits>

#include "lanes.h"
#include "lds_dma.h"
#include "ops_kernels.h"
#include "rows8.h"
#include "stage_ops.h"

namespace stg {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) u32x4 *lds16;

constexpr int kTile = 16;     // rows of a tile
constexpr int kStep = 32;     // k (rank) of an MFMA

__device__ __forceinline__ void load8(const void *p, size_t e, int type, float v[8]) {
    if (type == STAGE_F32) {
        const float4 *f = reinterpret_cast<const float4 *>(static_cast<const float *>(p) + e);
        const float4 x = f[0], y = f[1];
        v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
        v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
    } else {
        const bf16x8_t b = *reinterpret_cast<const bf16x8_t *>(static_cast<const uint16_t *>(p) + e);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = (float)b[j];
    }
}
// Eight elements of a hi/lo pair, whose sum is exact.
__device__ __forceinline__ void load8_pair(const void *p, size_t at, float v[8]) {
    const uint16_t *const h = static_cast<const uint16_t *>(p) + at;
    const bf16x8_t hi = *reinterpret_cast<const bf16x8_t *>(h), lo = *reinterpret_cast<const bf16x8_t *>(h + 32);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (float)hi[j] + (float)lo[j];
}
// x as a sum of bf16 terms, each the nearest to what the ones before leave: three terms hold all 24 bits.
template <int TERMS>
__device__ __forceinline__ void split_terms8(const float v[8], bf16x8_t t[TERMS]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        float x = v[j];
#pragma unroll
        for (int i = 0; i < TERMS; ++i) {
            t[i][j] = (__bf16)x;
            x -= (float)t[i][j];
        }
    }
}

// Whether some are not finite.
__device__ __forceinline__ bool not_finite(const f32x4_t &v) {
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) most = max(most, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    return most >= 0x7F800000u;
}

__device__ __forceinline__ int rank_of(const AdapterArgs &a, int id) {
    return a.ranks ? min(max(a.ranks[id], 0), a.max_rank) : a.max_rank;
}
// The adapters of a tile's rows: lane r < 16 has row r's (-1: none, or of rank 0); `first` has a bit for the first row
// of each.  Every lane of the wavefront must be active.
struct TileIds {
    int id, rank;
    unsigned first;
    __device__ __forceinline__ void load(const AdapterArgs &a, int row0) {
        const int lane = __lane_id(), row = row0 + (lane & 15);
        id = row < a.rows ? a.ids[row] : -1;
        rank = (unsigned)id < (unsigned)a.n_adapters ? rank_of(a, id) : 0;
        if (rank == 0) id = -1;
        bool again = id < 0;
#pragma unroll
        for (int i = 0; i < 15; ++i) again |= (i < (lane & 15)) & (__builtin_amdgcn_readlane(id, i) == id);
        first = (unsigned)__builtin_amdgcn_ballot_w64(!again) & 0xFFFFu;
    }
};

struct AdapterPlan {
    int wave_k;           // k of a wavefront (a multiple of kStep, up to kWaveK); four of them side by side are a slice
    int slices;
    int groups;           // workgroups that share a tile and slice's (adapter, 16 of its ranks) items
};

// Four of a row's t over n of its k by products of whole numbers: of an infinity, or an x too large for bf16, the terms are
// none (inf - inf).
__device__ __forceinline__ f32x4_t whole_sums(const AdapterArgs &a, int row, int id, int j0, int k0, int n) {
    asm volatile("" : "+v"(id), "+v"(row));   // (nothing of it is worked out ahead, and kept in registers)
    f32x4_t v = {0.f, 0.f, 0.f, 0.f};
    const uint16_t *const w = a.a + ((size_t)id * a.max_rank + j0) * a.k;
#pragma unroll 1
    for (int k = k0; k < min(a.k, k0 + n); k += 8) {
        float x[8], y[8];
        if (a.x_pair) load8_pair(a.x, (size_t)row * a.x_ld + pair_at(k), x);
        else load8(a.x, (size_t)row * a.x_ld + k, STAGE_F32, x);
        bool nan = false;   // (with one the rest does not matter)
#pragma unroll
        for (int j = 0; j < 8; ++j) nan |= x[j] != x[j];
        if (nan) return f32x4_t{NAN, NAN, NAN, NAN};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            load8(w, (size_t)i * a.k + k, STAGE_BF16, y);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i] = fmaf(x[j], y[j], v[i]);
        }
    }
    return v;
}

// t of a tile over a slice of k: a wavefront holds its k of x as operand fragments and takes one item (adapter, 16 of its
// ranks) after the other, its rows of A copied into LDS one item ahead; the four wavefronts' sums meet in LDS.
constexpr int kWaveK = 128;
template <int TERMS>
__global__ __launch_bounds__(256) void adapter_down_kernel(AdapterArgs a, AdapterPlan pl) {
    constexpr int TYPE = TERMS == 1 ? STAGE_BF16 : STAGE_F32, STEPS = kWaveK / kStep, CH = kWaveK / 8;
    constexpr int STAGE = 16 * kWaveK * 2, COPIES = STAGE / 1024;
    __shared__ __align__(1024) char ring_lds[4 * 2 * STAGE];
    __shared__ f32x4_t sums[2][4][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, lq = lane >> 4;
    const int row0 = kTile * blockIdx.x, slice = blockIdx.y;
    const int k0 = (4 * slice + wave) * pl.wave_k, k1 = min(a.k, k0 + pl.wave_k);   // the wavefront's (none: k1 <= k0)
    const uint32_t ring = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)ring_lds + wave * 2 * STAGE;
    // x: lane's chunks of eight k, a row's side by side
    float v[STEPS][8];
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        const int e = 64 * i + lane, r = e / CH, k = k0 + e % CH * 8;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
        if (k < k1 && row0 + r < a.rows) {
            if (TYPE == STAGE_F32 && a.x_pair) load8_pair(a.x, (size_t)(row0 + r) * a.x_ld + pair_at(k), v[i]);
            else load8(a.x, (size_t)(row0 + r) * a.x_ld + k, TYPE, v[i]);
        }
    }
    TileIds t;
    t.load(a, row0);
    // the items of this workgroup: every groups-th
    unsigned left = t.first;
    int jb = 0;
    struct Item { int id, jb; };
    auto next = [&]() {
        Item it{-1, 0};
        if (left) {
            const int at = __builtin_ctz(left);
            it = {__builtin_amdgcn_readlane(t.id, at), jb};
            if (16 * ++jb >= __builtin_amdgcn_readlane(t.rank, at)) {
                left &= left - 1;
                jb = 0;
            }
        }
        return it;
    };
    auto skip = [&](int n) {
        for (int i = 0; i < n && left; ++i) next();
    };
    // chunk c of row r at [r][c ^ r]: every 16 lanes of a fragment's read meet distinct banks
    auto copy = [&](const Item &it, int stage) {
        if (it.id < 0 || k0 >= k1) return;
        const uint16_t *const w = a.a + ((size_t)it.id * a.max_rank + 16 * it.jb) * a.k + k0;
        const int last = a.max_rank - 1 - 16 * it.jb;
#pragma unroll
        for (int i = 0; i < COPIES; ++i) {
            const int e = 64 * i + lane, r = e / CH, c = (e % CH) ^ r;
            // (rows past the last rank: that one; k past the last: the wavefront's first, cleared below)
            const uint32_t k = k0 + 8 * c < k1 ? 8 * c : 0;
            dma16(2 * ((uint32_t)min(r, last) * (uint32_t)a.k + k), w, ring + stage * STAGE + 1024 * i);
        }
    };
    skip(blockIdx.z);
    Item it = next();
    copy(it, 0);
    // x's fragments, term by term by way of the other stage: chunk c of row r at place 16 (c % 4) + (r ^ c % 16) of step c / 4
    bf16x8_t x[STEPS][TERMS];
#pragma unroll
    for (int n = 0; n < TERMS; ++n) {
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            const int e = 64 * i + lane, r = e / CH, c = e % CH;
            bf16x8_t b;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                b[j] = (__bf16)v[i][j];
                v[i][j] -= (float)b[j];
            }
            *(lds16)(ring + STAGE + c / 4 * 1024 + 16 * (16 * (c % 4) + (r ^ (c & 15)))) = __builtin_bit_cast(u32x4, b);
        }
        asm volatile("" ::: "memory");
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
            x[s][n] = __builtin_bit_cast(bf16x8_t, *(lds16)(ring + STAGE + s * 1024 + 16 * (16 * lq + (l16 ^ ((4 * s + lq) & 15)))));
        asm volatile("" ::: "memory");
    }
    const bool tail = k1 - k0 < kWaveK;
    for (int turn = 0; it.id >= 0; ++turn) {
        skip(pl.groups - 1);
        const Item after = next();
        wait_lgkm<0>();   // the other stage's last readers are done
        asm volatile("" ::: "memory");
        copy(after, (turn + 1) & 1);
        if (after.id >= 0) wait_vm<COPIES>();   // (a wavefront without k waits for nothing)
        else wait_vm<0>();
        asm volatile("" ::: "memory");
        f32x4_t d = {0.f, 0.f, 0.f, 0.f};
        if (k0 < k1) {
            const uint32_t st = ring + (turn & 1) * STAGE + l16 * (CH * 16);
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                u32x4 f = *(lds16)(st + 16 * ((4 * s + lq) ^ l16));
                if (tail && k0 + kStep * s + 8 * lq >= k1) f = u32x4{0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < TERMS; ++i)
                    d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, f), x[s][i], d, 0, 0, 0);
            }
        }
        sums[turn & 1][wave][lane] = d;
        wait_lgkm<0>();   // (the copies under way stay so across the barrier)
        lds_barrier();
        // rank 16 jb + 4 lq + i of row l16
        const int j0 = 16 * it.jb + 4 * lq;
        if (wave == (turn & 3) && t.id == it.id && j0 < a.max_rank) {
            const f32x4_t *const p = &sums[turn & 1][0][lane];
            f32x4_t v = ((p[0] + p[64]) + p[128]) + p[192];
            if constexpr (TERMS > 1) {
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = j0 + i < t.rank ? v[i] : 0.f;   // (past the rank A holds anything)
            }
            if (__builtin_expect(TERMS > 1 && not_finite(v), 0)) v = whole_sums(a, row0 + l16, it.id, j0, 4 * slice * pl.wave_k, 4 * pl.wave_k);
            *reinterpret_cast<f32x4_t *>(a.part + ((size_t)slice * a.rows + row0 + l16) * a.max_rank + j0) = v;
        }
        it = after;
    }
}

__device__ __forceinline__ const uint16_t *uniform(const uint16_t *p, int lane) {
    const uint64_t t = (uint64_t)(uintptr_t)p;
    const uint32_t low = __builtin_amdgcn_readlane((uint32_t)t, lane), high = __builtin_amdgcn_readlane((uint32_t)(t >> 32), lane);
    return reinterpret_cast<const uint16_t *>((uintptr_t)((uint64_t)high << 32 | low));
}
// Eight elements of a row of B from j0 on, 8 bytes at a time (rows of a multiple of four); past the rank: any.
__device__ __forceinline__ u32x4 load_ranks(const uint16_t *w, int j0, int rank) {
    const uint2 x = *reinterpret_cast<const uint2 *>(w + (j0 < rank ? j0 : 0)), y = *reinterpret_cast<const uint2 *>(w + (j0 + 4 < rank ? j0 + 4 : 0));
    return u32x4{x.x, x.y, y.x, y.y};
}
// Elements past the rank become 0.
__device__ __forceinline__ u32x4 cut_ranks(u32x4 v, int j0, int rank) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        v[j] = j0 + 2 * j < rank ? v[j] : 0;
        v[j] = j0 + 2 * j + 1 < rank ? v[j] : v[j] & 0xFFFFu;
    }
    return v;
}

// 16 columns of a row's B t, likewise, from column `col` on.
__device__ __forceinline__ void whole_outputs(const AdapterArgs &a, int slices, int row, int id, int col, f32x4_t (&v)[4]) {
    asm volatile("" : "+v"(id), "+v"(row));
    const int rank = rank_of(a, id);
    const float scale = a.scales ? a.scales[id] : 1.f;
#pragma unroll
    for (int m = 0; m < 4; ++m) v[m] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int j = 0; j < rank; ++j) {
        float t = 0.f;
#pragma unroll 1
        for (int s = 0; s < slices; ++s) t += a.part[((size_t)s * a.rows + row) * a.max_rank + j];
        t *= scale;
#pragma unroll
        for (int i = 0; i < 16; ++i)   // (columns past the last: that one)
            v[i / 4][i % 4] = fmaf(t, __uint_as_float((uint32_t)a.b[((size_t)id * a.n + min(col + i, a.n - 1)) * a.max_rank + j] << 16), v[i / 4][i % 4]);
        if (t != t) break;
    }
}

// At most n memory operations of this wavefront still under way (fewer where n is between two of the counts).
__device__ __forceinline__ void wait_most(int n) {
    if (n >= 8) {
        if (n >= 16) n >= 20 ? wait_vm<20>() : wait_vm<16>();
        else n >= 12 ? wait_vm<12>() : n >= 10 ? wait_vm<10>() : wait_vm<8>();
    } else if (n >= 4) {
        n >= 6 ? wait_vm<6>() : wait_vm<4>();
    } else {
        n >= 2 ? wait_vm<2>() : n == 1 ? wait_vm<1>() : wait_vm<0>();
    }
}

// A workgroup: a tile and blocks of 64 columns of out, a wavefront each.  A block's items are the tile's adapters, and
// of each up to 64 ranks at a time; B's of the next item (and base's of a block with its first) are copied into LDS
// while one is multiplied; the loop has no load of another kind, whose wait would take in the copies.  WAYS
// wavefronts share the blocks, and so may workgroups (grid z), each with every so manieth adapter, whose rows it writes (the
// first also those without one): 16 rows of 16 adapters, 64 blocks, 4 workgroups to a block take
// 6.6 us, one 9.6.  A lane has 16 neighbouring columns of a row: MFMA m's row i is column 16 (i / 4) + 4 m + i % 4 of the block.
//
// A turn is as long as the latency of its own instructions, of one or two wavefronts per SIMD, so it has few: the items,
// the same for every block, are listed once, an item per lane; t's fragments stay in registers.
constexpr int kCols = 64, kRanks = 64;
template <int TYPE>
struct UpLds {   // a wavefront's: S stages of B (by the adapters' rank), S of base
    static constexpr int S = 2, E = TYPE == STAGE_F32 ? 4 : 2, Y_STAGE = kTile * kCols * E, YCOPIES = Y_STAGE / 1024;
    static constexpr int b_stage(int max_rank) { return kCols * 2 * (max_rank > 32 ? 64 : max_rank > 16 ? 32 : 16); }
    static constexpr int bytes(int max_rank) { return S * (b_stage(max_rank) + Y_STAGE); }
};
template <int TYPE, int WAYS, int T_STEPS>
__global__ __launch_bounds__(256, T_STEPS * kStep <= kRanks ? 3 : 1) void adapter_up_kernel(AdapterArgs a, AdapterPlan pl, int blocks_per_group) {
    using L = UpLds<TYPE>;
    constexpr int S = L::S, E = L::E, YCOPIES = L::YCOPIES, YCH = kCols * E / 16;
    extern __shared__ __align__(1024) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, lq = lane >> 4;
    const int row0 = kTile * blockIdx.y, R = a.max_rank, b_stage = L::b_stage(R);
    const int row = row0 + l16;
    TileIds t;
    t.load(a, row0);
    // this wavefront's items, an item per lane: B's first place for it, how many of the adapter's ranks are left, and
    // the adapter; and whether the lane's row is its to write
    const int way = wave % WAYS + WAYS * blockIdx.z, ways = WAYS * gridDim.z;
    const uint16_t *item_b = nullptr;
    int item_ranks = 0, item_id = -1, n_items = 0, seen = 0;
    bool write = t.id < 0 && way == 0;
    for (unsigned left = t.first; left; left &= left - 1, ++seen)
        if (seen % ways == way) {
            const int at = __builtin_ctz(left), id = __builtin_amdgcn_readlane(t.id, at), rank = __builtin_amdgcn_readlane(t.rank, at);
            const int mine = lane - n_items;
            if (mine >= 0 && kRanks * mine < rank) {
                item_b = a.b + (size_t)id * a.n * R + kRanks * mine;
                item_ranks = rank - kRanks * mine;
                item_id = id;
            }
            n_items += (rank + kRanks - 1) / kRanks;
            write |= t.id == id;
        }
    write &= row < a.rows;
    const bool any = __builtin_amdgcn_ballot_w64(write) != 0, wide = R % 8 == 0;
    const int n_blocks = (a.n + kCols - 1) / kCols;
    const int end = blockIdx.z > 0 && !any ? 0 : min(n_blocks, (int)(blockIdx.x + 1) * blocks_per_group);
    if (n_items == 0) n_items = 1;   // (of no rank: base to out)
    const uint32_t ring = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds + wave * L::bytes(R);
    const uint32_t y_ring = ring + S * b_stage;

    struct Place { int nb, slot, item, ranks, copies; };   // block and its place in y_ring, item, its ranks, its copies
    auto fill = [&](Place &p) { p.ranks = p.nb < end ? __builtin_amdgcn_readlane(item_ranks, p.item) : 0; };
    auto advance = [&](Place &p) {
        if (++p.item == n_items) {
            p.item = 0;
            p.nb += 4 / WAYS;
            p.slot ^= 1;
        }
        fill(p);
    };
    // log2 of the 16-byte chunks that the item's rows have in LDS: 2, 4 or 8
    auto log_chunks = [](int ranks) { return ranks <= 16 ? 1 : ranks <= 32 ? 2 : 3; };
    // whether they are all of the adapter's ranks
    auto exact = [](int ranks) { return (ranks == 16) | (ranks == 32) | (ranks >= 64); };
    // chunk c of row r lies at c ^ place(r): every 16 lanes of a fragment's read meet distinct banks (two chunks: pairs)
    auto place = [](int r, int lc) { return ((r & 3) | (r >> 4 & 3) << 2) >> (4 - lc); };
    auto y_place = [](int r) { return YCH == 16 ? r : r >> 1; };   // (likewise, of 16 rows of base)
    // where instruction i of base's copies reads, for a whole block
    uint32_t y_from[YCOPIES];
#pragma unroll
    for (int i = 0; i < YCOPIES; ++i) {
        const int e = 64 * i + lane, r = e / YCH, c = (e % YCH) ^ y_place(r);
        y_from[i] = E * (uint32_t)min(r, a.rows - 1 - row0) * (uint32_t)a.base_ld + 16 * c;
    }
    // copies of B for whole blocks of all ranks: instruction i has rows (64 >> LC) i + lane / 2^LC, of which place() takes
    // i (LC 1, 2) or lane / 16 % 2 and i / 2 (LC 3)
    auto copy_whole = [&](auto log, const uint16_t *w, uint32_t at) {
        constexpr int LC = decltype(log)::value;
        const uint32_t rows = 2 * (uint32_t)(lane >> LC) * R;
        const uint32_t c = 16 * ((lane & ((1 << LC) - 1)) ^ (LC == 3 ? lane >> 4 & 1 : 0));
#pragma unroll
        for (int i = 0; i < 1 << LC; ++i)
            dma16((c ^ (16 * (LC == 3 ? i / 2 * 2 : i))) + rows, w + (size_t)i * (64 >> LC) * R, at + 1024 * i);
    };
    using One = std::integral_constant<int, 1>;
    using Two = std::integral_constant<int, 2>;
    using Three = std::integral_constant<int, 3>;
    auto copy = [&](Place &p, uint32_t at) {
        p.copies = 0;
        if (p.nb >= end) return;
        const bool whole = kCols * (p.nb + 1) <= a.n;
        if (p.item == 0) {
            p.copies = YCOPIES;
            const char *const from = static_cast<const char *>(a.base) + E * ((size_t)row0 * a.base_ld + (size_t)kCols * p.nb);
#pragma unroll
            for (int i = 0; i < YCOPIES; ++i) {
                uint32_t y = y_from[i];
                if (!whole) {   // columns past the last: the first
                    const int e = 64 * i + lane, c = ((e % YCH) ^ y_place(e / YCH)) * (16 / E);
                    if (kCols * p.nb + c >= a.n) y -= E * c;
                }
                dma16(y, from, y_ring + (p.slot * YCOPIES + i) * 1024);
            }
        }
        if (p.ranks == 0 || !wide) return;
        const int lc = log_chunks(p.ranks), n = 1 << lc;
        p.copies += n;
        const uint16_t *const w = uniform(item_b, p.item) + (size_t)kCols * p.nb * R;
        if (whole & exact(p.ranks)) {
            if (lc == 3) copy_whole(Three{}, w, at);
            else if (lc == 2) copy_whole(Two{}, w, at);
            else copy_whole(One{}, w, at);
            return;
        }
        const int last = a.n - 1 - kCols * p.nb;
#pragma unroll 1
        for (int i = 0; i < n; ++i) {
            const int e = 64 * i + lane, r = e >> lc, c = (e & ((1 << lc) - 1)) ^ place(r, lc);
            // (rows past the last column: that one; chunks past the rank: the first, cut below)
            dma16(2 * ((uint32_t)min(r, last) * R + (8 * c < p.ranks ? 8 * c : 0)), w, at + 1024 * i);
        }
    };
    // the fragments' first addresses: row 16 (l16 / 4) + l16 % 4, chunk lq
    const int fr = 16 * (l16 >> 2) + (l16 & 3);
    auto frag_from = [&](int lc) { return (uint32_t)(16 * ((fr << lc) + ((lq & ((1 << lc) - 1)) ^ place(fr, lc)))); };
    const uint32_t from1 = frag_from(1), from2 = frag_from(2), from3 = frag_from(3);
    Place p0{(int)blockIdx.x * blocks_per_group + wave / WAYS, 0, 0, 0, 0};
    fill(p0);
    // t as operand fragments: the slices added, a row's ranks by neighbouring lanes, into LDS (where the first wavefront's
    // second stage will be; of more ranks, where the first ones will be)
    constexpr bool EARLY = kStep * T_STEPS <= kRanks;
    if (EARLY) copy(p0, ring);
    float *const t_lds = reinterpret_cast<float *>(lds + (EARLY ? b_stage : 0));
    const int quads = R / 4, trow = R + 4;
    for (int e = threadIdx.x; e < kTile * quads; e += 256) {
        const int r = e / quads, j = e % quads * 4;
        const float *const p = a.part + (size_t)min(row0 + r, a.rows - 1) * R + j;
        f32x4_t v = {0.f, 0.f, 0.f, 0.f};
        for (int s0 = 0; s0 < pl.slices; s0 += 8) {
            f32x4_t u[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) u[i] = *reinterpret_cast<const f32x4_t *>(p + (size_t)min(s0 + i, pl.slices - 1) * a.rows * R);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (s0 + i < pl.slices) v += u[i];
        }
        *reinterpret_cast<f32x4_t *>(t_lds + r * trow + j) = v;
    }
    const float scale = a.scales && t.id >= 0 ? a.scales[t.id] : 1.f;
    wait_lgkm<0>();
    lds_barrier();
    bf16x8_t x[T_STEPS][3];
#pragma unroll
    for (int s = 0; s < T_STEPS; ++s) {
        float v[8];
        const int j0 = kStep * s + 8 * lq;
#pragma unroll
        for (int h = 0; h < 8; h += 4) {
            const f32x4_t u = *reinterpret_cast<const f32x4_t *>(t_lds + l16 * trow + min(j0 + h, R - 4));
#pragma unroll
            for (int j = 0; j < 4; ++j) v[h + j] = j0 + h + j < t.rank ? u[j] * scale : 0.f;   // (others' are not looked at)
        }
        split_terms8<3>(v, x[s]);
    }
    wait_lgkm<0>();
    lds_barrier();
    if (!EARLY) copy(p0, ring);
    f32x4_t d[4], sum[4];   // of the adapter; of the row's adapter
    int stores = 0, first_step = 0;   // stores of the turn before, behind the copies of p0's
    uint32_t at = ring;
    while (p0.nb < end) {
        Place p1 = p0;
        advance(p1);
        const uint32_t other = at == ring ? ring + b_stage : ring;
        wait_lgkm<0>();   // its last readers are done
        asm volatile("" ::: "memory");
        copy(p1, other);
        wait_most(p1.copies + stores);
        asm volatile("" ::: "memory");
        stores = 0;
        const int id = __builtin_amdgcn_readlane(item_id, p0.item);
        u32x4 f[2][4];
        if (!wide) {
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    f[e][m] = u32x4{0, 0, 0, 0};
                    if (kStep * e < p0.ranks)
                        f[e][m] = load_ranks(uniform(item_b, p0.item) + (size_t)min(kCols * p0.nb + fr + 4 * m, a.n - 1) * R, kStep * e + 8 * lq, p0.ranks);
                }
        } else if (p0.ranks > 32) {
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int m = 0; m < 4; ++m) f[e][m] = *(lds16)(at + (from3 ^ 64 * e) + 512 * m);
        } else {
            const uint32_t from = at + (p0.ranks > 16 ? from2 : from1), by = p0.ranks > 16 ? 256 : 128;
            const uint32_t keep = p0.ranks > 16 || lq < 2 ? ~0u : 0u;   // (of two chunks, for the lanes that have them)
#pragma unroll
            for (int m = 0; m < 4; ++m) f[0][m] = *(lds16)(from + by * m) & u32x4{keep, keep, keep, keep};
        }
        if (!wide | !exact(p0.ranks)) {
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int m = 0; m < 4; ++m)
                    if (kStep * e < p0.ranks) f[e][m] = cut_ranks(f[e][m], kStep * e + 8 * lq, p0.ranks);
        }
        if (first_step == 0) {
#pragma unroll
            for (int m = 0; m < 4; ++m) d[m] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }
#pragma unroll
        for (int s = 0; s < T_STEPS; s += 2) {
            if (s != first_step) continue;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                if (kStep * e >= p0.ranks || s + e >= T_STEPS) break;
#pragma unroll
                for (int i = 0; i < 3; ++i)
#pragma unroll
                    for (int m = 0; m < 4; ++m)
                        d[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, f[e][m]), x[s + e < T_STEPS ? s + e : 0][i], d[m], 0, 0, 0);
            }
        }
        const bool last = p0.ranks <= kRanks;   // of the adapter
        first_step = last ? 0 : first_step + 2;
        if (last && t.id == id) {
#pragma unroll
            for (int m = 0; m < 4; ++m) sum[m] = d[m];
        }
        if (p1.nb != p0.nb) {   // the block's last
            if (any) stores = E;
            const int c0 = kCols * p0.nb + 16 * lq;
            if (write && c0 < a.n) {
                if (__builtin_expect((t.id >= 0) & (not_finite(sum[0]) | not_finite(sum[1]) | not_finite(sum[2]) | not_finite(sum[3])), 0))
                    whole_outputs(a, pl.slices, row, t.id, c0, sum);
                const uint32_t from = y_ring + p0.slot * L::Y_STAGE + l16 * (16 * YCH);
#pragma unroll
                for (int h = 0; h < 2; ++h) {   // eight columns
                    float y[8];
                    if constexpr (TYPE == STAGE_F32) {
#pragma unroll
                        for (int g = 0; g < 2; ++g) {
                            const f32x4_t u = __builtin_bit_cast(f32x4_t, *(lds16)(from + 16 * ((4 * lq + 2 * h + g) ^ y_place(l16))));
#pragma unroll
                            for (int i = 0; i < 4; ++i) y[4 * g + i] = u[i];
                        }
                    } else {
                        const bf16x8_t u = __builtin_bit_cast(bf16x8_t, *(lds16)(from + 16 * ((2 * lq + h) ^ y_place(l16))));
#pragma unroll
                        for (int i = 0; i < 8; ++i) y[i] = (float)u[i];
                    }
                    if (t.id >= 0) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) y[i] += sum[2 * h + i / 4][i % 4];
                    }
                    if (c0 + 8 * h < a.n) store8(a.out, (size_t)row * a.out_ld + c0 + 8 * h, TYPE, y);
                }
            }
        }
        p0 = p1;
        at = other;
    }
}

AdapterPlan adapter_plan(const AdapterArgs &a) {
    AdapterPlan p{};
    const long tiles = (a.rows + kTile - 1) / kTile, want = 2L * device_compute_units();
    const int quarter = ((a.k + 3) / 4 + kStep - 1) / kStep * kStep;
    p.wave_k = quarter < kWaveK ? quarter : kWaveK;
    p.slices = (a.k + 4 * p.wave_k - 1) / (4 * p.wave_k);
    // workgroups enough to fill the chip twice: a tile's items apart
    const long items = (long)(a.n_adapters < kTile ? a.n_adapters : kTile) * ((a.max_rank + 15) / 16);
    const long have = tiles * p.slices, groups = (want + have - 1) / have;
    p.groups = (int)(groups < items ? groups : items);
    return p;
}

template <int TYPE>
hipError_t launch_up(const AdapterArgs &a, const AdapterPlan &p, unsigned tiles, hipStream_t st) {
    const int blocks = (a.n + kCols - 1) / kCols, lds = 4 * UpLds<TYPE>::bytes(a.max_rank);
    // workgroups: as many as run at once (by LDS; the registers are held to those of three, 4001 rows of rank 32 58 -> 52 us)
    const long want = (lds > 80 * 1024 ? 1L : lds > 53 * 1024 ? 2L : 3L) * device_compute_units();
    // few tiles: the wavefronts share a block's adapters; many: a block each
    const bool shared = p.groups > 1 && a.n_adapters >= 4;
    const int least = shared ? 1 : 4;
    long per = ((long)blocks * tiles + want - 1) / want;
    per = (per + least - 1) / least * least;
    // fewer workgroups than run at once: more of them share a block's adapters, four of which each takes
    const long most = ((a.n_adapters < kTile ? a.n_adapters : kTile) + 3) / 4, room = want / ((long)blocks * tiles);
    const dim3 grid((unsigned)((blocks + per - 1) / per), tiles, (unsigned)(!shared || room < 2 ? 1 : room < most ? room : most));
    auto launch = [&](auto ways, auto steps) -> hipError_t {
        auto *const kernel = adapter_up_kernel<TYPE, decltype(ways)::value, decltype(steps)::value>;
        STG_LAUNCH(kernel, grid, dim3(256), lds, st, a, p, (int)per);
        return hipGetLastError();
    };
    using One = std::integral_constant<int, 1>;
    using Four = std::integral_constant<int, 4>;
    using Few = std::integral_constant<int, kRanks / kStep>;
    using Most = std::integral_constant<int, STAGE_OPS_MAX_RANK / kStep>;
    if (a.max_rank <= kRanks) return shared ? launch(Four{}, Few{}) : launch(One{}, Few{});
    return shared ? launch(Four{}, Most{}) : launch(One{}, Most{});
}

__global__ __launch_bounds__(256) void adapter_rows_kernel(SeqAdapters of, int rows, int rows_per_seq, int *ids) {
    const int row = blockIdx.x * 256 + threadIdx.x;
    if (row < rows) ids[row] = of.id[row / rows_per_seq];
}

}  // namespace

size_t adapter_workspace(const AdapterArgs &a) {
    return a.rows <= 0 ? 0 : (size_t)adapter_plan(a).slices * a.rows * a.max_rank * sizeof(float);
}

hipError_t launch_adapter_add(const AdapterArgs &a, hipStream_t st) {
    if (a.rows <= 0) return hipSuccess;
    const AdapterPlan p = adapter_plan(a);
    const unsigned tiles = (a.rows + kTile - 1) / kTile;
    if (tiles > 65535 || p.slices > 65535) return hipErrorInvalidValue;
    const dim3 down(tiles, p.slices, p.groups);
    if (a.type == STAGE_F32) {
        STG_LAUNCH(adapter_down_kernel<3>, down, dim3(256), 0, st, a, p);
        return launch_up<STAGE_F32>(a, p, tiles, st);
    } else {
        STG_LAUNCH(adapter_down_kernel<1>, down, dim3(256), 0, st, a, p);
        return launch_up<STAGE_BF16>(a, p, tiles, st);
    }
}

hipError_t launch_adapter_rows(const SeqAdapters &of, int rows, int rows_per_seq, int *ids, hipStream_t st) {
    if (rows <= 0) return hipSuccess;
    STG_LAUNCH(adapter_rows_kernel, dim3((rows + 255) / 256), dim3(256), 0, st, of, rows, rows_per_seq, ids);
    return hipGetLastError();
}

}  // namespace stg
