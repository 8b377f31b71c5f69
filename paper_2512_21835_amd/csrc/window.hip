// Grouped-query attention with a sliding window and sinks over the paged cache.
//
// The keys that a block of consecutive rows may see are two runs of cache pages: the first tokens' (sinks) and
// the window's, which meet where the window reaches back to the sinks.  The kernels walk that list of pages and
// mask inside the pages at its ends.
//
// window_split: rows in blocks of 16 columns (G query heads of a KV head x 16 / G positions), the pages cut
// over workgroups and their wavefronts, states joined at the end (window_merge where the workgroups are several).
#include "lanes.h"
#include "lds_dma.h"
#include "ops_kernels.h"
#include "pair.h"
#include "stage_ops.h"

namespace stg {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef const __attribute__((address_space(4))) int *const_ints;
typedef __attribute__((address_space(3))) u32x4 *lds16;
typedef __attribute__((address_space(3))) s16x4_t *lds8;
typedef __attribute__((address_space(3))) float *lds4;

constexpr int kPage = kBlockTokens;
constexpr float kLog2e = 1.4426950408889634f;

// The pages that rows at positions first .. last see: pages 0 .. sink - 1, then from, from + 1, ...; n in all.
struct Span {
    int end;          // keys from here on are seen by no row
    int sink, from, n;
    __device__ __forceinline__ int page(int u) const { return u < sink ? u : from + u - sink; }
};
__device__ __forceinline__ Span span_of(const WindowArgs &a, int first, int last) {
    Span s;
    s.end = min(last + 1, a.rows.max_len);
    s.sink = (max(0, min(a.sinks, s.end)) + kPage - 1) / kPage;
    s.from = max(max(0, first - a.window + 1) / kPage, s.sink);
    s.n = s.sink + max(0, (s.end + kPage - 1) / kPage - s.from);
    if (s.end <= 0) s.n = 0;
    return s;
}
__device__ __forceinline__ bool sees(const WindowArgs &a, int pos, int key) {
    return key <= pos && key < a.rows.max_len && (key > pos - a.window || key < a.sinks);
}
// Whether rows at positions first .. last all see keys k0 .. k0 + n - 1.
__device__ __forceinline__ bool all_see(const WindowArgs &a, int first, int last, int k0, int n) {
    return k0 + n - 1 <= first && k0 + n <= a.rows.max_len && (k0 > last - a.window || k0 + n <= a.sinks);
}

__device__ __forceinline__ float load_elem(const void *p, size_t e, int type) {
    if (type == STAGE_F32) return static_cast<const float *>(p)[e];
    return __uint_as_float((uint32_t)static_cast<const uint16_t *>(p)[e] << 16);
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
__device__ __forceinline__ void store4(void *p, size_t e, int type, float4 v) {
    if (type == STAGE_F32) {
        *reinterpret_cast<float4 *>(static_cast<float *>(p) + e) = v;
    } else {
        typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
        *reinterpret_cast<bf16x4 *>(static_cast<uint16_t *>(p) + e) = bf16x4{(__bf16)v.x, (__bf16)v.y, (__bf16)v.z, (__bf16)v.w};
    }
}
// o / l; a row that saw no key is 0.
__device__ __forceinline__ float4 quotient(float4 o, float l) {
    if (l == 0.f) return make_float4(0.f, 0.f, 0.f, 0.f);
    return make_float4(o.x / l, o.y / l, o.z / l, o.w / l);
}

// Term t of x as a sum of bf16 terms, each the nearest to what the ones before leave: three terms hold all 24 bits.
template <int TERMS>
__device__ __forceinline__ void split_terms(float x, __bf16 t[TERMS]) {
#pragma unroll
    for (int i = 0; i < TERMS; ++i) {
        t[i] = (__bf16)x;
        x -= (float)t[i];
    }
}

// The LDS image of a cache page: K rows, then V rows, as they lie in the cache, with the 16-byte chunks of each row
// permuted (by the copies' lane addresses) so that the fragments' reads meet distinct banks.
template <int D, bool F32>
struct PageLds {
    static constexpr int ROW = D * (F32 ? 4 : 2), HALF = kPage * ROW, BYTES = 2 * HALF;
    static constexpr int COPIES = BYTES / 1024;                  // instructions of 64 x 16 bytes
    // a page's share per wavefront: as many in flight as 32 KB hold (16 KB of 64-wide bf16 heads)
    static constexpr int STAGES = F32 && D == 128 ? 2 : 4;
    static constexpr int KEYS = 1024 / ROW, CH = ROW / 16;       // keys per copy, chunks per row
    __device__ static int kx(int key) { return ROW == 128 ? (key >> 1) & 7 : key & 15; }
    __device__ static int vx(int key) {
        if (F32) return (key >> 2 & 3) << 2;
        return ROW == 128 ? (key >> 1 & 3) << 1 : (key & 7) << 1;
    }
};

// One wavefront's attention of 16 columns over its pages.  Everything of it is the wavefront's own: no barrier.
//
// S^T = K Q^T: lane l holds keys 4 (l / 16) + i of the page for column l % 16, which is the layout of the operand P^T of
// O^T += V^T P^T, so probabilities stay in registers; o[b][i]: d 16 b + 4 (l / 16) + i of column l % 16.  bf16 cache:
// 16x16x32 and 16x16x16 MFMAs, V^T by transposing reads, q and p as TERMS bf16 terms.  fp32 cache: 16x16x4 fp32 MFMAs, k
// index l / 16 of step (v, c) being d 16 v + 4 (l / 16) + c, so that K is read 16 bytes at a time.
template <int D, bool F32, int TERMS>
struct Columns {
    using L = PageLds<D, F32>;
    bf16x8_t q[F32 ? 1 : TERMS][D / 32];
    float qf[F32 ? D / 4 : 1];
    f32x4_t o[D / 16];
    float m, l;       // of column l % 16; l: of the lane's keys only
    int pos;          // of the column's row; -1: no row

    __device__ __forceinline__ void init(const WindowArgs &a, size_t q_at, bool valid) {
        const int lane = __lane_id(), lq = lane >> 4;
        m = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int b = 0; b < D / 16; ++b) o[b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        if constexpr (F32) {
#pragma unroll
            for (int v = 0; v < D / 16; ++v) {
                float x[4] = {0.f, 0.f, 0.f, 0.f};
                if (valid) load4(a.q, q_at + 16 * v + 4 * lq, a.type, x);
#pragma unroll
                for (int c = 0; c < 4; ++c) qf[4 * v + c] = x[c];
            }
        } else {
#pragma unroll
            for (int s = 0; s < D / 32; ++s) {
                float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                if (valid) {
                    load4(a.q, q_at + 32 * s + 8 * lq, a.type, x);
                    load4(a.q, q_at + 32 * s + 8 * lq + 4, a.type, x + 4);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    __bf16 t[TERMS];
                    split_terms<TERMS>(x[j], t);
#pragma unroll
                    for (int i = 0; i < TERMS; ++i) q[i][s][j] = t[i];
                }
            }
        }
    }

    // lds: the page's image; k0: its first key; masked: some column does not see all of it; rows: of the block
    // (positions first .. first + rows - 1)
    __device__ __forceinline__ void add(const WindowArgs &a, uint32_t lds, int k0, bool masked, int first, int rows) {
        const int lane = __lane_id(), l16 = lane & 15, lq = lane >> 4;
        f32x4_t sc = {0.f, 0.f, 0.f, 0.f}, s1 = sc;
        const uint32_t kr = lds + l16 * L::ROW;
        if constexpr (F32) {
#pragma unroll
            for (int v = 0; v < D / 16; ++v) {
                const f32x4_t k = __builtin_bit_cast(f32x4_t, *(lds16)(kr + 16 * ((4 * v + lq) ^ L::kx(l16))));
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    if (c & 1) s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[c], qf[4 * v + c], s1, 0, 0, 0);
                    else sc = __builtin_amdgcn_mfma_f32_16x16x4f32(k[c], qf[4 * v + c], sc, 0, 0, 0);
                }
            }
        } else {
#pragma unroll
            for (int s = 0; s < D / 32; ++s) {
                const bf16x8_t k = __builtin_bit_cast(bf16x8_t, *(lds16)(kr + 16 * ((4 * s + lq) ^ L::kx(l16))));
#pragma unroll
                for (int t = 0; t < TERMS; ++t) {
                    if (t & 1) s1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[t][s], s1, 0, 0, 0);
                    else sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[t][s], sc, 0, 0, 0);
                }
            }
        }
        const float scale = a.scale * kLog2e;   // scores in base 2
        float p[4], top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            p[i] = (sc[i] + s1[i]) * scale;
            if (masked && !sees(a, pos, k0 + 4 * lq + i)) p[i] = -INFINITY;
            top = fmaxf(top, p[i]);
        }
        top = fmaxf(top, lane_xor(top, 16));
        top = fmaxf(top, lane_xor(top, 32));
        top = fmaxf(top, m);
        const float ref = top == -INFINITY ? 0.f : top, alpha = __builtin_amdgcn_exp2f(m - ref);
        m = top;
        l *= alpha;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            p[i] = __builtin_amdgcn_exp2f(p[i] - ref);
            l += p[i];
        }
        if (__builtin_amdgcn_ballot_w64(alpha != 1.f) != 0) {   // some column's maximum moved
#pragma unroll
            for (int b = 0; b < D / 16; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[b][i] *= alpha;
        }
        const uint32_t vr = lds + L::HALF;
        if (masked) hide(a, vr, k0, first, rows, p);
        if constexpr (F32) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int key = 4 * lq + i;
#pragma unroll
                for (int b = 0; b < D / 16; ++b) {
                    const int c = 4 * b + l16 / 4;
                    const float v = *(lds4)(vr + key * L::ROW + 16 * (c ^ L::vx(key)) + 4 * (l16 & 3));
                    o[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, p[i], o[b], 0, 0, 0);
                }
            }
        } else {
            s16x4_t pt[TERMS];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                __bf16 t[TERMS];
                split_terms<TERMS>(p[i], t);
#pragma unroll
                for (int j = 0; j < TERMS; ++j) pt[j][i] = __builtin_bit_cast(short, t[j]);
            }
            // a transposing read gives 16 lanes the 4 keys x 16 d that they point at (lane i: key i / 4, d 4 (i % 4) ..
            // + 3) column-wise: lane i all keys of d i
            const int key = 4 * lq + l16 / 4;
            const uint32_t at = vr + key * L::ROW + 8 * (l16 & 1);
#pragma unroll
            for (int b = 0; b < D / 16; ++b) {
                const s16x4_t v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds8)(at + 16 * ((2 * b + (l16 >> 1 & 1)) ^ L::vx(key))));
#pragma unroll
                for (int j = 0; j < TERMS; ++j) o[b] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(v, pt[j], o[b], 0, 0, 0);
            }
        }
    }

    // The V of a place that a column does not see must not meet the matrix instructions if it is not finite (0 x
    // inf).  Rows of V that no row of the block sees become 0.  Where rows see different keys, elements that are
    // not finite are added by hand for the columns that see them, and become 0 too: nothing else changes a bit.
    __device__ __forceinline__ void hide(const WindowArgs &a, uint32_t vr, int k0, int first, int rows, const float p[4]) {
        const int lane = __lane_id(), last = first + rows - 1;
        constexpr int N = L::HALF / 1024;
        bool odd = false;
#pragma unroll
        for (int c = 0; c < N; ++c) {
            const int at = 64 * c + lane, key = k0 + at / L::CH;
            // (a key between two rows' windows is in one of them: the rows are neighbours)
            if (!sees(a, last, key) && !(key <= last && sees(a, max(first, key), key))) {
                *(lds16)(vr + 16 * at) = u32x4{0, 0, 0, 0};
            } else if (rows > 1) {
                u32x4 v = *(lds16)(vr + 16 * at);
                odd = odd || zero_odd(v);
            }
        }
        if (rows > 1 && __builtin_amdgcn_ballot_w64(odd) != 0) {
            add_odd(a, vr, k0, p);
#pragma unroll
            for (int c = 0; c < N; ++c) {
                u32x4 v = *(lds16)(vr + 16 * (64 * c + lane));
                zero_odd(v);
                *(lds16)(vr + 16 * (64 * c + lane)) = v;
            }
        }
        asm volatile("" ::: "memory");   // (the reads behind this are of what it wrote)
    }
    // Clears the elements of v that are not finite; whether there are any.
    __device__ __forceinline__ static bool zero_odd(u32x4 &v) {
        bool odd = false;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool high = (v[j] & 0x7F800000u) == 0x7F800000u, low = !F32 && (v[j] & 0x7F80u) == 0x7F80u;
            odd = odd || high || low;
            if (high) v[j] &= F32 ? 0u : 0xFFFFu;
            if (low) v[j] &= 0xFFFF0000u;
        }
        return odd;
    }
    __device__ __forceinline__ void add_odd(const WindowArgs &a, uint32_t vr, int k0, const float p[4]) {
        const int lane = __lane_id(), l16 = lane & 15, lq = lane >> 4;
#pragma unroll 1
        for (int key = 0; key < kPage; ++key) {
            const float mine = key & 2 ? (key & 1 ? p[3] : p[2]) : (key & 1 ? p[1] : p[0]);
            const float w = __shfl(mine, 16 * (key / 4) + l16, 64);
            if (!sees(a, pos, k0 + key)) continue;
#pragma unroll
            for (int b = 0; b < D / 16; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int d = 16 * b + 4 * lq + i, c = d * (F32 ? 4 : 2) / 16;
                    const uint32_t at = vr + key * L::ROW + 16 * (c ^ L::vx(key)) + d * (F32 ? 4 : 2) % 16;
                    float v;
                    if constexpr (F32) v = *(lds4)at;
                    else v = __uint_as_float((uint32_t)*(const __attribute__((address_space(3))) uint16_t *)at << 16);
                    if (!(fabsf(v) < INFINITY)) o[b][i] = fmaf(w, v, o[b][i]);
                }
        }
    }
};

struct SplitPlan {
    int log_g, blocks_per_seq;   // query heads per KV head (log2); row blocks per sequence
    int pages;                   // per wavefront
    int splits;                  // workgroups that share a block's pages
};

template <int D, bool F32, int TERMS>
__global__ __launch_bounds__(256) void window_split(WindowArgs a, SplitPlan pl) {
    using L = PageLds<D, F32>;
    constexpr int S = L::STAGES, OLD = D + 4;    // (padding: the columns' stores meet distinct banks)
    constexpr int RING = 4 * S * L::BYTES, JOIN = 4 * 16 * OLD * 4 + 4 * 32 * 4;
    __shared__ __align__(1024) char lds[RING > JOIN ? RING : JOIN];
    const int lane = threadIdx.x & 63, l16 = lane & 15, lq = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hkv = a.n_kv_heads, g = blockIdx.x % hkv, block = blockIdx.x / hkv, split = blockIdx.y;
    const int bq = 16 >> pl.log_g, seq_i = block / pl.blocks_per_seq, t0 = block % pl.blocks_per_seq * bq;
    const OpRows::Seq seq = a.rows.seq(seq_i);
    const int n = min(seq.n, a.rows.max_rows);
    if (t0 >= n) return;
    const int rows = min(bq, n - t0), first = seq.pos0 + t0, last = first + rows - 1;
    const Span sp = span_of(a, first, last);
    const int beg = (split * 4 + wave) * pl.pages, end = min(beg + pl.pages, sp.n);
    if (split > 0 && split * 4 * pl.pages >= sp.n) return;   // (split 0 stays: a row that sees nothing is written)

    const uint32_t ring = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds + wave * S * L::BYTES;
    const size_t head = (size_t)kPage * L::ROW, block_bytes = (size_t)2 * hkv * head;
    const char *const pool = static_cast<const char *>(a.pool) + g * head;
    auto block_of = [&](int u) { return ((const_ints)(uintptr_t)seq.table)[sp.page(u)]; };
    auto known = [&](int b) { return (unsigned)b < (unsigned)a.rows.n_blocks; };
    auto copy = [&](int u, int b) {
        const char *const k = pool + (size_t)(known(b) ? b : 0) * block_bytes;
        const uint32_t st = ring + u % S * L::BYTES;
        const int r = lane / L::CH, c = lane % L::CH;
#pragma unroll
        for (int i = 0; i < L::COPIES / 2; ++i) {
            const int key = i * L::KEYS + r;
            dma16(key * L::ROW + 16 * (c ^ L::kx(key)), k, st + 1024 * i);
            dma16(key * L::ROW + 16 * (c ^ L::vx(key)), k + hkv * head, st + L::HALF + 1024 * i);
        }
    };
    int blk[S];   // of pages u, u + 1, ...: known before they are needed
#pragma unroll
    for (int i = 0; i < S; ++i) blk[i] = beg + i < end ? block_of(beg + i) : -1;
#pragma unroll
    for (int i = 0; i < S - 1; ++i)
        if (beg + i < end) copy(beg + i, blk[i]);

    Columns<D, F32, TERMS> cols;
    const int t = l16 >> pl.log_g, h = (g << pl.log_g) + (l16 & ((1 << pl.log_g) - 1));
    const size_t row = seq.first + t0 + min(t, rows - 1);
    cols.pos = t < rows ? first + t : -1;
    cols.init(a, row * a.q_ld + (size_t)h * D, t < rows);

    for (int u = beg; u < end; ++u) {
        const int b = blk[0];
        wait_lgkm<0>();   // the stage's last readers are done
        asm volatile("" ::: "memory");
        const int left = end - 1 - u;   // pages behind this one
        if (left >= S - 1) {
            copy(u + S - 1, blk[S - 1]);
            wait_vm<(S - 1) * L::COPIES>();
        } else if (S > 3 && left == 2) {
            wait_vm<2 * L::COPIES>();
        } else if (S > 2 && left == 1) {
            wait_vm<L::COPIES>();
        } else {
            wait_vm<0>();
        }
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < S - 1; ++i) blk[i] = blk[i + 1];
        blk[S - 1] = u + S < end ? block_of(u + S) : -1;
        if (!known(b)) continue;
        const int k0 = sp.page(u) * kPage;
        cols.add(a, ring + u % S * L::BYTES, k0, !all_see(a, first, last, k0, kPage), first, rows);
    }

    // the wavefronts' states meet in LDS
    float l = cols.l;
    l += lane_xor(l, 16);
    l += lane_xor(l, 32);
    __syncthreads();
    float *const so = reinterpret_cast<float *>(lds), *const sm = so + 4 * 16 * OLD;   // [wave][col][OLD]; [wave][m, l][col]
#pragma unroll
    for (int b = 0; b < D / 16; ++b)
        *reinterpret_cast<f32x4_t *>(so + (wave * 16 + l16) * OLD + 16 * b + 4 * lq) = cols.o[b];
    if (lq == 0) {
        sm[wave * 32 + l16] = cols.m;
        sm[wave * 32 + 16 + l16] = l;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < 16 * (D / 4); e += 256) {
        const int col = e / (D / 4), d = 4 * (e % (D / 4)), ct = col >> pl.log_g;
        if (ct >= rows) continue;
        float M = -INFINITY, sum = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) M = fmaxf(M, sm[w * 32 + col]);
        const float ref = M == -INFINITY ? 0.f : M;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = __builtin_amdgcn_exp2f(sm[w * 32 + col] - ref);
            const f32x4_t v = *reinterpret_cast<const f32x4_t *>(so + (w * 16 + col) * OLD + d);
            sum = fmaf(f, sm[w * 32 + 16 + col], sum);
            o.x = fmaf(f, v.x, o.x);
            o.y = fmaf(f, v.y, o.y);
            o.z = fmaf(f, v.z, o.z);
            o.w = fmaf(f, v.w, o.w);
        }
        const size_t r = seq.first + t0 + ct;
        const int hc = (g << pl.log_g) + (col & ((1 << pl.log_g) - 1));
        if (pl.splits == 1) {
            store4(a.out, r * a.out_ld + (size_t)hc * D + d, a.type, quotient(o, sum));
        } else {
            const size_t st = (r * a.n_q_heads + hc) * pl.splits + split;
            float *const ml = a.part + (size_t)a.rows.rows * a.n_q_heads * pl.splits * D;
            *reinterpret_cast<float4 *>(a.part + st * D + d) = o;
            if (d == 0) *reinterpret_cast<float2 *>(ml + 2 * st) = make_float2(M, sum);
        }
    }
}

// Joins a row's states: a wavefront per (row, query head), 64 / (D / 4) states at a time, then the lanes' sums.
template <int D>
__global__ __launch_bounds__(256) void window_merge(WindowArgs a, SplitPlan pl) {
    constexpr int CG = D / 4, SL = 64 / CG;
    const int lane = threadIdx.x & 63, cg = lane % CG, sl = lane / CG;
    const int h = blockIdx.y * 4 + (threadIdx.x >> 6), seq_i = blockIdx.x / a.rows.max_rows, t = blockIdx.x % a.rows.max_rows;
    if (h >= a.n_q_heads) return;
    const OpRows::Seq seq = a.rows.seq(seq_i);
    const int n = min(seq.n, a.rows.max_rows);
    if (t >= n) return;
    const int bq = 16 >> pl.log_g, t0 = t / bq * bq, first = seq.pos0 + t0;
    const Span sp = span_of(a, first, first + min(bq, n - t0) - 1);
    const int states = max(1, (sp.n + 4 * pl.pages - 1) / (4 * pl.pages));
    const size_t row = seq.first + t, st = (row * a.n_q_heads + h) * pl.splits;
    const float *const po = a.part + st * D + 4 * cg;
    const float2 *const ml = reinterpret_cast<const float2 *>(a.part + (size_t)a.rows.rows * a.n_q_heads * pl.splits * D) + st;
    float m = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    auto join = [&](float m1, float l1, float4 o1) {
        const float top = fmaxf(m, m1), ref = top == -INFINITY ? 0.f : top;
        const float r = __builtin_amdgcn_exp2f(m - ref), w = __builtin_amdgcn_exp2f(m1 - ref);
        m = top;
        l = fmaf(w, l1, l * r);
        o = make_float4(fmaf(w, o1.x, o.x * r), fmaf(w, o1.y, o.y * r), fmaf(w, o1.z, o.z * r), fmaf(w, o1.w, o.w * r));
    };
#pragma unroll 4
    for (int s = sl; s < states; s += SL) {
        const float2 x = ml[s];
        join(x.x, x.y, *reinterpret_cast<const float4 *>(po + (size_t)s * D));
    }
#pragma unroll
    for (int x = CG; x < 64; x *= 2) {
        const float m1 = lane_xor(m, x), l1 = lane_xor(l, x);
        const float4 o1 = make_float4(lane_xor(o.x, x), lane_xor(o.y, x), lane_xor(o.z, x), lane_xor(o.w, x));
        join(m1, l1, o1);
    }
    if (sl == 0) store4(a.out, row * a.out_ld + (size_t)h * D + 4 * cg, a.type, quotient(o, l));
}

SplitPlan split_plan(const WindowArgs &a) {
    SplitPlan p{};
    while (a.n_kv_heads << p.log_g < a.n_q_heads) ++p.log_g;
    const int bq = 16 >> p.log_g, most = a.rows.max_rows < a.rows.rows ? a.rows.max_rows : a.rows.rows;
    p.blocks_per_seq = (most + bq - 1) / bq;
    // pages of the longest list: all, or the sinks' and the window's of a block (which may start inside a page)
    const long all = (a.rows.max_len + kPage - 1) / kPage;
    const long listed = (a.sinks + kPage - 1) / kPage + ((long)a.window + bq + 2 * kPage - 3) / kPage;
    const long pages = listed < all ? listed : all;
    const long blocks = (long)a.rows.n_seqs * p.blocks_per_seq * a.n_kv_heads;
    const long groups = 2L * device_compute_units();
    const long splits = blocks >= groups ? 1 : (groups + blocks - 1) / blocks;
    p.pages = (int)((pages + 4 * splits - 1) / (4 * splits));
    p.splits = (int)((pages + 4L * p.pages - 1) / (4L * p.pages));
    return p;
}

template <int D, bool F32, int TERMS>
hipError_t launch_split(const WindowArgs &a, hipStream_t st) {
    const SplitPlan p = split_plan(a);
    const long blocks = (long)a.rows.n_seqs * p.blocks_per_seq * a.n_kv_heads;
    if (blocks > 0x7FFFFFFF || p.splits > 65535) return hipErrorInvalidValue;
    STG_LAUNCH((window_split<D, F32, TERMS>), dim3((unsigned)blocks, p.splits), dim3(256), 0, st, a, p);
    if (p.splits > 1) {
        const long rows = (long)a.rows.n_seqs * a.rows.max_rows;
        STG_LAUNCH((window_merge<D>), dim3((unsigned)rows, (a.n_q_heads + 3) / 4), dim3(256), 0, st, a, p);
    }
    return hipGetLastError();
}

}  // namespace

size_t window_workspace(const WindowArgs &a) {
    if (a.rows.rows <= 0) return 0;
    const SplitPlan p = split_plan(a);
    return p.splits == 1 ? 0 : (size_t)a.rows.rows * a.n_q_heads * p.splits * (a.head_dim + 2) * sizeof(float);
}

hipError_t launch_window_attention(const WindowArgs &a, hipStream_t st) {
    if (a.rows.rows <= 0) return hipSuccess;
    const bool f32 = a.kv_type == STAGE_F32, exact = a.type == STAGE_F32;
#define STG_WINDOW_CASE(D)                                                 \
    if (a.head_dim == D)                                                   \
        return f32 ? launch_split<D, true, 1>(a, st)                       \
                   : exact ? launch_split<D, false, 3>(a, st) : launch_split<D, false, 1>(a, st);
    STG_WINDOW_CASE(64) STG_WINDOW_CASE(128)
#undef STG_WINDOW_CASE
    return hipErrorInvalidValue;
}

}  // namespace stg
