// Low-rank adapters of many requests beside a shared projection: out = base + scale B (A x), a pair (A, B) per row.
//
// Two launches.  Down: t = A x over slices of k, whose sums go to the workspace; up: the slices added, out = base + scale B
// t.  Both take tiles of 16 rows as the columns of 16x16x32 MFMAs and loop over the adapters that occur in the tile; a
// product of another row's adapter is dropped with its column, so no row's values meet another's.  Bound by bytes: A
// and B of the adapters present (decode), x, base and out (prompts).  fp32 operands enter as the exact sum of three
// bf16 terms.
#include "lanes.h"
#include "ops_kernels.h"
#include "stage_ops.h"

namespace stg {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

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
__device__ __forceinline__ void store8(void *p, size_t e, int type, const float v[8]) {
    if (type == STAGE_F32) {
        float4 *f = reinterpret_cast<float4 *>(static_cast<float *>(p) + e);
        f[0] = make_float4(v[0], v[1], v[2], v[3]);
        f[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
        bf16x8_t b;
#pragma unroll
        for (int j = 0; j < 8; ++j) b[j] = (__bf16)v[j];
        *reinterpret_cast<bf16x8_t *>(static_cast<uint16_t *>(p) + e) = b;
    }
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

// The adapters of a tile's rows: lane r < 16 has row r's (-1: none, or of rank 0); `first` has a bit for the first row
// of each.  Every lane of the wavefront must be active.
struct TileIds {
    int id, rank;
    unsigned first;
    __device__ __forceinline__ void load(const AdapterArgs &a, int row0) {
        const int lane = __lane_id(), row = row0 + (lane & 15);
        id = row < a.rows ? a.ids[row] : -1;
        rank = (unsigned)id < (unsigned)a.n_adapters ? a.ranks ? min(max(a.ranks[id], 0), a.max_rank) : a.max_rank : 0;
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

// t of a tile over a slice of k: a wavefront holds its k of x as operand fragments and takes one item (adapter, 16 of its
// ranks) after the other, A straight from memory (16 rows x 64 bytes per instruction, all of an item's under way
// together, the next item's behind them); the four wavefronts' sums meet in LDS.
constexpr int kWaveK = 256;
template <int TERMS>
__global__ __launch_bounds__(256) void adapter_down_kernel(AdapterArgs a, AdapterPlan pl) {
    constexpr int TYPE = TERMS == 1 ? STAGE_BF16 : STAGE_F32, STEPS = kWaveK / kStep;
    __shared__ f32x4_t sums[2][4][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, lq = lane >> 4;
    const int row0 = kTile * blockIdx.x, slice = blockIdx.y;
    const int k0 = (4 * slice + wave) * pl.wave_k + 8 * lq, k1 = min(a.k, (4 * slice + wave + 1) * pl.wave_k);   // the lane's
    float v[STEPS][8];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[s][j] = 0.f;
        if (k0 + kStep * s < k1 && row0 + l16 < a.rows) load8(a.x, (size_t)(row0 + l16) * a.x_ld + k0 + kStep * s, TYPE, v[s]);
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
    auto load = [&](const Item &it, u32x4 f[STEPS]) {
        const uint16_t *const w = a.a + ((size_t)max(it.id, 0) * a.max_rank + min(16 * it.jb + l16, a.max_rank - 1)) * a.k + k0;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            f[s] = u32x4{0, 0, 0, 0};
            if (it.id >= 0 && k0 + kStep * s < k1) f[s] = *reinterpret_cast<const u32x4 *>(w + kStep * s);
        }
    };
    skip(blockIdx.z);
    Item it = next();
    u32x4 f[STEPS];
    load(it, f);
    bf16x8_t x[STEPS][TERMS];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) split_terms8<TERMS>(v[s], x[s]);
    for (int turn = 0; it.id >= 0; ++turn) {
        skip(pl.groups - 1);
        const Item after = next();
        u32x4 g[STEPS];
        load(after, g);
        f32x4_t d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int i = 0; i < TERMS; ++i)
                d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, f[s]), x[s][i], d, 0, 0, 0);
        sums[turn & 1][wave][lane] = d;
        __syncthreads();
        // rank 16 jb + 4 lq + i of row l16
        if (wave == (turn & 3) && t.id == it.id && 16 * it.jb + 4 * lq < a.max_rank) {
            const f32x4_t *const p = &sums[turn & 1][0][lane];
            *reinterpret_cast<f32x4_t *>(a.part + ((size_t)slice * a.rows + row0 + l16) * a.max_rank + 16 * it.jb + 4 * lq) =
                ((p[0] + p[64]) + p[128]) + p[192];
        }
        it = after;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) f[s] = g[s];
    }
}

// Eight elements of a row of B from j0 on, of `have` (0: any eight: they are not looked at).
__device__ __forceinline__ bf16x8_t load_ranks(const uint16_t *w, int j0, int have, bool wide) {
    u32x4 v;
    if (wide) {
        v = *reinterpret_cast<const u32x4 *>(w + (j0 < have ? j0 : 0));
    } else {   // (rows of a multiple of four)
        const uint2 x = *reinterpret_cast<const uint2 *>(w + (j0 < have ? j0 : 0)), y = *reinterpret_cast<const uint2 *>(w + (j0 + 4 < have ? j0 + 4 : 0));
        v = u32x4{x.x, x.y, y.x, y.y};
    }
    return __builtin_bit_cast(bf16x8_t, v);
}
// Elements past the rank become 0.
__device__ __forceinline__ bf16x8_t cut_ranks(bf16x8_t b, int j0, int rank) {
    u32x4 v = __builtin_bit_cast(u32x4, b);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        v[j] = j0 + 2 * j < rank ? v[j] : 0;
        v[j] = j0 + 2 * j + 1 < rank ? v[j] : v[j] & 0xFFFFu;
    }
    return __builtin_bit_cast(bf16x8_t, v);
}

// A workgroup: a tile and 32-column blocks of out.  A wavefront takes BLOCKS of them at a time, with IDS of the tile's
// adapters at a time, all loads of both under way together.  WAYS wavefronts share the blocks, each with every
// WAYS-th adapter, whose rows it writes (the first also those without one).  A lane has eight neighbouring columns of a
// row: MFMA m's row i is column 8 (i / 4) + 4 m + i % 4 of the block.
template <int TYPE, int WAYS, int IDS, int BLOCKS>
__global__ __launch_bounds__(256) void adapter_up_kernel(AdapterArgs a, AdapterPlan pl, int blocks_per_group) {
    extern __shared__ __align__(16) char lds[];
    bf16x8_t *const ts = reinterpret_cast<bf16x8_t *>(lds);   // t as operand fragments, [rank step][term][lane]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, lq = lane >> 4;
    const int row0 = kTile * blockIdx.y, R = a.max_rank, rank_steps = (R + kStep - 1) / kStep;
    const int row = row0 + l16;
    TileIds t;
    t.load(a, row0);
    const float scale = a.scales && t.id >= 0 ? a.scales[t.id] : 1.f;
    for (int s = wave; s < rank_steps; s += 4) {
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        const int j0 = kStep * s + 8 * lq;
#pragma unroll
        for (int h = 0; h < 8; h += 4) {
            if (j0 + h >= t.rank) continue;
            const float *p = a.part + (size_t)row * R + j0 + h;
            f32x4_t sum = *reinterpret_cast<const f32x4_t *>(p);
#pragma unroll 8
            for (int sl = 1; sl < pl.slices; ++sl) sum += *reinterpret_cast<const f32x4_t *>(p + (size_t)sl * a.rows * R);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[h + j] = j0 + h + j < t.rank ? sum[j] * scale : 0.f;
        }
        bf16x8_t b[3];
        split_terms8<3>(v, b);
#pragma unroll
        for (int i = 0; i < 3; ++i) ts[(s * 3 + i) * 64 + lane] = b[i];
    }
    __syncthreads();
    // this wavefront's adapters, and whether this lane's row is its to write
    const int way = wave % WAYS;
    unsigned ids = 0;
    int seen = 0;
    bool write = t.id < 0 && way == 0;
    for (unsigned left = t.first; left; left &= left - 1, ++seen)
        if (seen % WAYS == way) {
            const int at = __builtin_ctz(left);
            ids |= 1u << at;
            write |= (t.id >= 0) & (__builtin_amdgcn_readlane(t.id, at) == t.id);
        }
    const bool wide = R % 8 == 0;
    const int n_blocks = (a.n + 31) / 32, end = min(n_blocks, (int)(blockIdx.x + 1) * blocks_per_group);
    // The blocks, for each the adapters, for each the steps of their ranks: one step's loads of B are under way while
    // the step before is multiplied (and base's of a block with those of its first step).
    struct Place { int nb, s, most; unsigned left; int id[IDS], rank[IDS]; };
    auto take = [&](Place &p) {   // the next adapters of p.left
        p.s = 0;
        p.most = 0;
#pragma unroll
        for (int u = 0; u < IDS; ++u) {   // (past the last: the first again, of rank 0)
            const int at = p.left ? __builtin_ctz(p.left) : 0;
            p.id[u] = p.left ? __builtin_amdgcn_readlane(t.id, at) : u ? p.id[0] : 0;
            p.rank[u] = p.left ? __builtin_amdgcn_readlane(t.rank, at) : 0;
            p.most = max(p.most, p.rank[u]);
            p.left &= p.left - 1;
        }
    };
    auto advance = [&](Place &p) {
        if (kStep * ++p.s < p.most) return;
        if (!p.left) {
            p.nb += 4 / WAYS * BLOCKS;
            p.left = ids;
        }
        take(p);
    };
    auto load_b = [&](const Place &p, bf16x8_t (&b)[IDS][BLOCKS][2]) {
        if (p.nb >= end || p.most == 0) return;
#pragma unroll
        for (int q = 0; q < BLOCKS; ++q) {
            const int c0 = 32 * (p.nb + q) + 8 * (l16 / 4) + l16 % 4;
#pragma unroll
            for (int u = 0; u < IDS; ++u)
#pragma unroll
                for (int m = 0; m < 2; ++m)
                    b[u][q][m] = load_ranks(a.b + ((size_t)p.id[u] * a.n + min(c0 + 4 * m, a.n - 1)) * R, kStep * p.s + 8 * lq, p.rank[u], wide);
        }
    };
    auto mine = [&](int nb) { return write && row < a.rows && 32 * nb + 8 * lq < a.n && nb < end; };
    auto load_y = [&](int nb, float (&y)[BLOCKS][8]) {
#pragma unroll
        for (int q = 0; q < BLOCKS; ++q)
            if (mine(nb + q)) load8(a.base, (size_t)row * a.base_ld + 32 * (nb + q) + 8 * lq, TYPE, y[q]);
    };
    Place at;
    at.nb = blockIdx.x * blocks_per_group + wave / WAYS * BLOCKS;
    at.left = ids;
    take(at);
    bf16x8_t b[IDS][BLOCKS][2];
    float y[BLOCKS][8];
    f32x4_t d[IDS][BLOCKS][2];
    load_b(at, b);
    load_y(at.nb, y);
    while (at.nb < end) {
        Place to = at;
        advance(to);
        bf16x8_t bn[IDS][BLOCKS][2];
        float yn[BLOCKS][8];
        load_b(to, bn);
        if (to.nb != at.nb) load_y(to.nb, yn);
        if (at.s == 0) {
#pragma unroll
            for (int u = 0; u < IDS; ++u)
#pragma unroll
                for (int q = 0; q < BLOCKS; ++q) d[u][q][0] = d[u][q][1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }
        bf16x8_t x[3];
#pragma unroll
        for (int i = 0; i < 3; ++i) x[i] = ts[(min(at.s, rank_steps - 1) * 3 + i) * 64 + lane];
#pragma unroll
        for (int u = 0; u < IDS; ++u) {
            if (kStep * at.s >= at.rank[u]) continue;
            const bool cut = kStep * (at.s + 1) > at.rank[u];
#pragma unroll
            for (int q = 0; q < BLOCKS; ++q)
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    const bf16x8_t f = cut ? cut_ranks(b[u][q][m], kStep * at.s + 8 * lq, at.rank[u]) : b[u][q][m];
#pragma unroll
                    for (int i = 0; i < 3; ++i) d[u][q][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, x[i], d[u][q][m], 0, 0, 0);
                }
        }
        if (to.s == 0) {   // the adapters' last step
#pragma unroll
            for (int u = 0; u < IDS; ++u)
                if (at.rank[u] > 0 && t.id == at.id[u]) {
#pragma unroll
                    for (int q = 0; q < BLOCKS; ++q)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            y[q][i] += d[u][q][0][i];
                            y[q][4 + i] += d[u][q][1][i];
                        }
                }
        }
        if (to.nb != at.nb) {   // and the block's
#pragma unroll
            for (int q = 0; q < BLOCKS; ++q)
                if (mine(at.nb + q)) store8(a.out, (size_t)row * a.out_ld + 32 * (at.nb + q) + 8 * lq, TYPE, y[q]);
#pragma unroll
            for (int q = 0; q < BLOCKS; ++q)
#pragma unroll
                for (int i = 0; i < 8; ++i) y[q][i] = yn[q][i];
        }
        at = to;
#pragma unroll
        for (int u = 0; u < IDS; ++u)
#pragma unroll
            for (int q = 0; q < BLOCKS; ++q)
#pragma unroll
                for (int m = 0; m < 2; ++m) b[u][q][m] = bn[u][q][m];
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
void launch_up(const AdapterArgs &a, const AdapterPlan &p, unsigned tiles, hipStream_t st) {
    const int blocks = (a.n + 31) / 32;
    const long want = 4L * device_compute_units();   // workgroups
    // few tiles: their wavefronts share the adapters, four at a time; many: four blocks at a time
    const bool shared = p.groups > 1 && a.n_adapters >= 4;
    const int least = shared ? 1 : 16;
    long per = ((long)blocks * tiles + want - 1) / want;
    per = (per + least - 1) / least * least;
    const size_t t_lds = (size_t)(a.max_rank + kStep - 1) / kStep * 3 * 1024;
    const dim3 grid((unsigned)((blocks + per - 1) / per), tiles);
    if (shared) STG_LAUNCH((adapter_up_kernel<TYPE, 4, 4, 1>), grid, dim3(256), t_lds, st, a, p, (int)per);
    else STG_LAUNCH((adapter_up_kernel<TYPE, 1, 1, 4>), grid, dim3(256), t_lds, st, a, p, (int)per);
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
        launch_up<STAGE_F32>(a, p, tiles, st);
    } else {
        STG_LAUNCH(adapter_down_kernel<1>, down, dim3(256), 0, st, a, p);
        launch_up<STAGE_BF16>(a, p, tiles, st);
    }
    return hipGetLastError();
}

}  // namespace stg
