// Grouped-query attention with a sliding window and sinks over the paged cache.
//
// The keys that a block of consecutive rows may see are two runs of cache pages: the first tokens' (sinks) and
// the window's, which meet where the window reaches back to the sinks.  The kernels walk that list of pages and
// mask inside the pages at its ends.
//
// window_split: rows in blocks of 16 columns (G query heads of a KV head x 16 / G positions), the pages cut
// over workgroups and their wavefronts, states joined at the end (window_merge where the workgroups are several).
// Bound by the cache's bytes: 64 single tokens of 64 heads over up to 4096 bf16 tokens each (8 KV heads, 727 MB)
// 138 us, 5.3 TB/s; a page costs a wavefront 1.2 us of dependent reads, products and softmax (fp32: 2.3), which
// is what shorter lists take (16 tokens of 32 heads over up to 1024 fp32 tokens, 83 MB: 38 us).
//
// window_tiles: prompts over a bf16 cache (over an fp32 cache: window_f32.hip).
#include <type_traits>

#include "lds_dma.h"
#include "window_rows.h"

namespace stg {
namespace {

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

// One wavefront's attention of 16 columns over its pages.  Everything of it is the wavefront's own: no barrier.  All
// fragments of a page's K, and later of its V, are read before the first of their MFMAs (read one by one between them, a
// wavefront alone on its SIMD waits for each: 3 us instead of 1 for a page of 128 fp32).
//
// S^T = K Q^T: lane l holds keys 4 (l / 16) + i of the page for column l % 16, which is the layout of the operand P^T of
// O^T += V^T P^T, so probabilities stay in registers; o[b][i]: d 16 b + 4 (l / 16) + i of column l % 16.  bf16 cache:
// 16x16x32 and 16x16x16 MFMAs, V^T by transposing reads, q as TERMS bf16 terms and p as p_terms().  fp32 cache: 16x16x4 fp32 MFMAs, k
// index l / 16 of step (v, c) being d 16 v + 4 (l / 16) + c, so that K is read 16 bytes at a time.
template <int D, bool F32, int TERMS>
struct Columns {
    using L = PageLds<D, F32>;
    static constexpr int PT = p_terms(TERMS);
    bf16x8_t q[F32 ? 1 : TERMS][D / 32];
    float qf[F32 ? D / 4 : 1];
    f32x4_t o[D / 16];
    float m, l;       // of column l % 16; l: of the lane's keys only
    int pos;          // of the column's row; -1: no row

    __device__ __forceinline__ void init(const WindowArgs &a, size_t q_at, bool valid) {
        if (a.type == STAGE_F32) init_of<STAGE_F32>(a, q_at, valid);
        else init_of<STAGE_BF16>(a, q_at, valid);
    }
    template <int TYPE>
    __device__ __forceinline__ void init_of(const WindowArgs &a, size_t q_at, bool valid) {
        const int lane = __lane_id(), lq = lane >> 4;
        m = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int b = 0; b < D / 16; ++b) o[b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        if constexpr (F32) {
#pragma unroll
            for (int v = 0; v < D / 16; ++v) {
                float x[4] = {0.f, 0.f, 0.f, 0.f};
                if (valid) load4(a.q, q_at + 16 * v + 4 * lq, TYPE, x);
#pragma unroll
                for (int c = 0; c < 4; ++c) qf[4 * v + c] = x[c];
            }
        } else {
#pragma unroll
            for (int s = 0; s < D / 32; ++s) {
                float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                if (valid) {
                    load4(a.q, q_at + 32 * s + 8 * lq, TYPE, x);
                    load4(a.q, q_at + 32 * s + 8 * lq + 4, TYPE, x + 4);
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

    // The columns whose state is not finite once more, key by key in fp32: of an infinity or a number too large for bf16 the
    // terms are none (inf - inf), and sums of large values pass the largest number.  pool: of the KV head.
    __device__ __forceinline__ void by_keys(const WindowArgs &a, const char *pool, const int *table, const Span &sp, int beg, int end,
                                            size_t q_at, bool valid) {
        uint32_t most = size_bits(l);
#pragma unroll
        for (int b = 0; b < D / 16; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) most = max(most, size_bits(o[b][i]));
        const int lane = __lane_id(), lq = lane >> 4;
        const uint64_t lanes = __builtin_amdgcn_ballot_w64(valid & (most >= 0x7F800000u));
        if (lanes == 0) return;
        const size_t head = (size_t)kPage * D;
        f32x4_t o2[D / 16];
        float m2 = -INFINITY, l2 = 0.f;
        const bool mine = lanes >> (lane & 15) & 0x0001000100010001ull;
        bool done = !mine;   // (a score that is NaN makes the column NaN, whatever follows)
#pragma unroll
        for (int b = 0; b < D / 16; ++b) o2[b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
        for (int u = beg * kPage; u < end * kPage && __builtin_amdgcn_ballot_w64(!done) != 0; ++u) {
            const int page = sp.page(u / kPage), key = page * kPage + u % kPage, block = ((const_ints)(uintptr_t)table)[page];
            if ((unsigned)block >= (unsigned)a.rows.n_blocks) continue;
            const size_t k = (size_t)block * 2 * a.n_kv_heads * head + u % kPage * D + 4 * lq, v = k + a.n_kv_heads * head;
            float w = 0.f;
#pragma unroll
            for (int b = 0; b < D / 16; ++b) {
                float x[4], y[4];
                load4(a.q, q_at + 16 * b + 4 * lq, a.type, x);
                load4(pool, k + 16 * b, F32 ? STAGE_F32 : STAGE_BF16, y);
#pragma unroll
                for (int i = 0; i < 4; ++i) w = fmaf(x[i], y[i], w);
            }
            w += lane_xor(w, 16);
            w += lane_xor(w, 32);
            w *= a.scale * kLog2e;
            const bool seen = sees(a, pos, key);
            const float to = seen & (w > m2) ? w : m2, ref = to == -INFINITY ? 0.f : to;
            const float alpha = __builtin_amdgcn_exp2f(m2 - ref);
            w = seen ? __builtin_amdgcn_exp2f(w - ref) * kRoom : 0.f;
            m2 = to;
            l2 = l2 * alpha + (lq == 0 ? w : 0.f);
#pragma unroll
            for (int b = 0; b < D / 16; ++b) {
                float x[4];
                load4(pool, v + 16 * b, F32 ? STAGE_F32 : STAGE_BF16, x);
#pragma unroll
                for (int i = 0; i < 4; ++i) o2[b][i] = o2[b][i] * alpha + (seen ? w * x[i] : 0.f);
            }
            done |= w != w;
            l2 = done ? NAN : l2;
        }
        if (mine) {
            m = m2 + kRoomBits;
            l = l2;
#pragma unroll
            for (int b = 0; b < D / 16; ++b) o[b] = o2[b];
        }
    }

    // lds: the page's image; k0: its first key; masked: some column does not see all of it; rows: of the block
    // (positions first .. first + rows - 1)
    __device__ __forceinline__ void add(const WindowArgs &a, uint32_t lds, int k0, bool masked, int first, int rows) {
        const int lane = __lane_id(), l16 = lane & 15, lq = lane >> 4;
        f32x4_t sc = {0.f, 0.f, 0.f, 0.f}, s1 = sc;
        const uint32_t kr = lds + l16 * L::ROW;
        if constexpr (F32) {
            f32x4_t k[D / 16];
#pragma unroll
            for (int v = 0; v < D / 16; ++v) k[v] = __builtin_bit_cast(f32x4_t, *(lds16)(kr + 16 * ((4 * v + lq) ^ L::kx(l16))));
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int v = 0; v < D / 16; ++v)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    if (c & 1) s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[v][c], qf[4 * v + c], s1, 0, 0, 0);
                    else sc = __builtin_amdgcn_mfma_f32_16x16x4f32(k[v][c], qf[4 * v + c], sc, 0, 0, 0);
                }
        } else {
            bf16x8_t k[D / 32];
#pragma unroll
            for (int s = 0; s < D / 32; ++s) k[s] = __builtin_bit_cast(bf16x8_t, *(lds16)(kr + 16 * ((4 * s + lq) ^ L::kx(l16))));
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int s = 0; s < D / 32; ++s)
#pragma unroll
                for (int t = 0; t < TERMS; ++t) {
                    if (t & 1) s1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[s], q[t][s], s1, 0, 0, 0);
                    else sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[s], q[t][s], sc, 0, 0, 0);
                }
        }
        const float scale = a.scale * kLog2e;   // scores in base 2
        float p[4], top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            p[i] = (sc[i] + s1[i]) * scale;
            p[i] = (!masked | sees(a, pos, k0 + 4 * lq + i)) ? p[i] : -INFINITY;
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
            float v[4][D / 16];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int b = 0; b < D / 16; ++b) {
                    const int key = 4 * lq + i, c = 4 * b + l16 / 4;
                    v[i][b] = *(lds4)(vr + key * L::ROW + 16 * (c ^ L::vx(key)) + 4 * (l16 & 3));
                }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int b = 0; b < D / 16; ++b) o[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[i][b], p[i], o[b], 0, 0, 0);
        } else {
            s16x4_t pt[PT];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                __bf16 t[PT];
                split_terms<PT>(p[i], t);
#pragma unroll
                for (int j = 0; j < PT; ++j) pt[j][i] = __builtin_bit_cast(short, t[j]);
            }
            // a transposing read gives 16 lanes the 4 keys x 16 d that they point at (lane i: key i / 4, d 4 (i % 4) ..
            // + 3) column-wise: lane i all keys of d i
            const int key = 4 * lq + l16 / 4;
            const uint32_t at = vr + key * L::ROW + 8 * (l16 & 1);
            s16x4_t v[D / 16];
#pragma unroll
            for (int b = 0; b < D / 16; ++b)
                v[b] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds8)(at + 16 * ((2 * b + (l16 >> 1 & 1)) ^ L::vx(key))));
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int b = 0; b < D / 16; ++b)
#pragma unroll
                for (int j = 0; j < PT; ++j) o[b] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(v[b], pt[j], o[b], 0, 0, 0);
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
            if (!(sees(a, last, key) | ((key <= last) & sees(a, max(first, key), key)))) {
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
    int log_g;       // query heads per KV head (log2)
    bool one_block;  // no sequence has more than one block of rows: block i is that of sequence i
    int blocks;      // of rows, over the KV heads: at most
    int pages;       // per wavefront
    int splits;      // workgroups that share a block's pages
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
    const int bq = 16 >> pl.log_g;
    OpRows::Seq seq;
    int t0 = 0;
    if (pl.one_block) {
        seq = uniform(a.rows.seq(block));
    } else {
        RowBlock rb;
        if (!rb.find(a, block, 4 - pl.log_g)) return;
        seq = rb.seq;
        t0 = rb.t0;
    }
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

    cols.by_keys(a, pool, seq.table, sp, beg, end, row * a.q_ld + (size_t)h * D, t < rows);

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
            const float f = __builtin_amdgcn_exp2f(sm[w * 32 + col] - ref) * kRoom;
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
            store4(a.out, r * a.out_ld + (size_t)hc * D + d, (long)r < a.pair_rows ? kPair : a.type, quotient(o, sum));
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
    const int h = blockIdx.y * 4 + (threadIdx.x >> 6), seq_i = a.rows.max_rows == 1 ? (int)blockIdx.x : a.rows.seq_of(blockIdx.x);
    if (h >= a.n_q_heads || seq_i >= a.rows.n_seqs) return;
    const OpRows::Seq seq = a.rows.seq(seq_i);
    const int n = min(seq.n, a.rows.max_rows), t = a.rows.max_rows == 1 ? 0 : (int)blockIdx.x - seq.first;
    if (t < 0 || t >= n) return;
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
    if (sl == 0) store4(a.out, row * a.out_ld + (size_t)h * D + 4 * cg, (long)row < a.pair_rows ? kPair : a.type, quotient(o, l));
}

// Blocks of `columns` columns that a call's rows fill, at most: of equal sequences, or no sequence adding more than one that is
// not full.
long row_blocks(const WindowArgs &a, long columns) {
    const long bq = columns * a.n_kv_heads / a.n_q_heads, seqs = a.rows.n_seqs < a.rows.rows ? a.rows.n_seqs : a.rows.rows;
    const long equal = (long)a.rows.n_seqs * ((a.rows.max_rows + bq - 1) / bq), ragged = a.rows.rows / bq + seqs;
    return (equal < ragged ? equal : ragged) * a.n_kv_heads;
}

SplitPlan split_plan(const WindowArgs &a) {
    SplitPlan p{};
    while (a.n_kv_heads << p.log_g < a.n_q_heads) ++p.log_g;
    const int bq = 16 >> p.log_g, most = a.rows.max_rows < a.rows.rows ? a.rows.max_rows : a.rows.rows;
    p.one_block = most <= bq;
    // pages of the longest list: all, or the sinks' and the window's of a block (which may start inside a page)
    const long all = (a.rows.max_len + kPage - 1) / kPage;
    const long listed = (a.sinks + kPage - 1) / kPage + ((long)a.window + bq + 2 * kPage - 3) / kPage;
    const long pages = listed < all ? listed : all;
    const long blocks = p.one_block ? (long)a.rows.n_seqs * a.n_kv_heads : row_blocks(a, 16);
    p.blocks = blocks > kMaxBlocks ? 0 : (int)blocks;
    // Workgroups that run at once: 128 KB of LDS each, 64 KB with bf16 heads of 64.  As many splits as fill one to four
    // rounds of them, whichever ends first: a round takes a wavefront's pages and the time of three to begin and end, the
    // joining launch as much (16 rows over 1024 fp32 tokens in two rounds 43 us, in one 38; 20 rows over 4096 bf16 tokens, 64
    // heads, in two rounds 80, in one of twice the length 90).  Four pages a wavefront at least.
    const long units = (a.head_dim == 64 && a.kv_type == STAGE_BF16 ? 2L : 1L) * device_compute_units();
    long least = 0;
    for (long rounds = 0; rounds <= 4; ++rounds) {
        const long want = rounds * units / (blocks > 0 ? blocks : 1), s = want < 1 ? 1 : want;
        long n = (pages + 4 * s - 1) / (4 * s);
        n = n < 4 ? 4 : n;
        const long splits = pages <= 4 * n ? 1 : (pages + 4 * n - 1) / (4 * n);
        const long cost = (blocks * splits + units - 1) / units * (n + 3) + (splits > 1 ? 3 : 0);
        if (rounds > 0 && cost >= least) continue;
        least = cost;
        p.pages = (int)n;
        p.splits = (int)splits;
    }
    return p;
}

template <int D, bool F32, int TERMS>
hipError_t launch_split(const WindowArgs &a, hipStream_t st) {
    const SplitPlan p = split_plan(a);
    if (p.blocks <= 0 || p.splits > 65535) return hipErrorInvalidValue;
    STG_LAUNCH((window_split<D, F32, TERMS>), dim3(p.blocks, p.splits), dim3(256), 0, st, a, p);
    if (p.splits > 1) {
        const int rows = a.rows.max_rows == 1 ? a.rows.n_seqs : a.rows.rows;
        STG_LAUNCH((window_merge<D>), dim3(rows, (a.n_q_heads + 3) / 4), dim3(256), 0, st, a, p);
    }
    return hipGetLastError();
}

// Prompts.  A workgroup: 128 columns = G heads x BQ = 128 / G consecutive rows of one sequence, one KV head; wavefront
// w the columns 32 w .. (column r: head r / BQ, row r % BQ).  K and V tiles of 32 keys (two pages) go straight into
// a ring of LDS stages, one barrier per tile.  S^T = K Q^T: lane l holds keys 8 (i / 4) + 4 (l / 32) + i % 4 of the tile for
// column l % 32, the k order of the operand P^T of O^T += V^T P^T; 32x32x16 MFMAs, q as TERMS bf16 terms, p as p_terms().
//
// In turn t a wavefront multiplies tile t + 1's K by Q and then tile t - 1's V by P while it takes the softmax of
// tile t: the three are independent, and the vector instructions of the softmax (as long as the MFMAs with one
// term of q) are laid between the MFMAs by hand.  Fragments are in registers half a turn before their MFMAs: V's are
// read under the scores, K's of the tile behind under the values.
//
// 4 x 2048 bf16 rows of 64 heads, window 1024: 357 us, 0.87 PFLOP/s of issued products (1.5 times the formula's, for the
// probabilities' second term; with one term, the output off by its own rounding once more, 286 us).  What is not loop is
// beginning (block search, page ids, first tiles: 3 to 4 us a workgroup), end, and the halves of tiles outside the window.
// 256 columns a workgroup (each wavefront 64) are slower: one wavefront per SIMD hides less than two.  fp32 rows issue three
// times the products: 12 prompts of up to 500 rows, window 512, 126 us.
template <int D>
struct TileLds {
    static constexpr int KEYS = 32, ROW = 2 * D, HALF = KEYS * ROW, BYTES = 2 * HALF, CH = ROW / 16;
    // tile t - 1 is read until the middle of turn t: its stage then takes tile t + S - 1
    static constexpr int STAGES = D == 128 ? 5 : 6;
    static constexpr int KPC = 1024 / ROW, COPIES = 8 / KPC;   // keys per copy; copies of K (and of V) per wavefront
    __device__ static int kx(int key) { return D == 128 ? key & 15 : (key >> 1) & 7; }
    __device__ static int vx(int key) { return D == 128 ? (key & 3) << 2 : (key & 2) << 1; }
};

// Clears the elements of eight bf16 that are not finite; whether there are any.
__device__ __forceinline__ bool clear_odd(u32x4 &v) {
    uint32_t odd = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t bad = ((v[j] & 0x7F807F80u) + 0x00800080u) & 0x80008000u;   // exponents all ones
        odd |= bad;
        v[j] &= ~((bad >> 15) * 0xFFFFu);
    }
    return odd != 0;
}

struct TilePlan {
    int log_g;
};

template <int D, int TERMS>
__global__ __launch_bounds__(256, TERMS == 1 ? 2 : 1) void window_tiles(WindowArgs a, TilePlan pl) {
    using L = TileLds<D>;
    constexpr int S = L::STAGES, KK = D / 16, NB = D / 32, KT = L::KEYS, PT = p_terms(TERMS);
    constexpr int TYPE = TERMS == 1 ? STAGE_BF16 : STAGE_F32;   // of q and out
    __shared__ __align__(1024) char lds[S * L::BYTES];
    const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hkv = a.n_kv_heads, g = blockIdx.x % hkv, log_bq = 7 - pl.log_g, bq = 1 << log_bq;
    RowBlock rb;
    if (!rb.find(a, blockIdx.x / hkv, log_bq)) return;
    const OpRows::Seq &seq = rb.seq;
    const int t0 = rb.t0, rows = rb.rows, first = rb.first, n_tiles = rb.n_tiles, last_page = rb.last_page;

    const uint32_t ring = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
    const size_t head = (size_t)kPage * L::ROW, block_bytes = (size_t)2 * hkv * head;
    const char *const pool = static_cast<const char *>(a.pool) + g * head;
    auto known = [&](int b) { return (unsigned)b < (unsigned)a.rows.n_blocks; };
    // Block ids of the tiles' pages, 64 (32 tiles) in a register of the wavefront, the next 64 under way: loads by
    // the scalar unit would have every wait for LDS wait for them, too.
    auto ids_from = [&](int t) { return seq.table[rb.page_at(t + lane / 2, lane & 1)]; };
    int ids = 0, more_ids = 0;
    if (n_tiles > 0) {
        ids = ids_from(0);
        more_ids = ids_from(32);
    }
    bool strange = __builtin_amdgcn_ballot_w64(!known(ids)) != 0;   // some page so far is not of the pool
    // the wavefront's share of a tile: 8 keys of K and of V, of one page, in 2 COPIES instructions
    const char *copy_from = nullptr;
    uint32_t copy_to = 0;
    auto copy_begin = [&](int t, uint32_t at) {   // (t ascending, each once)
        if (t > 0 && t % 32 == 0) {
            ids = more_ids;
            strange |= __builtin_amdgcn_ballot_w64(!known(ids)) != 0;
            more_ids = ids_from(t + 32);
        }
        const int b = __builtin_amdgcn_readlane(ids, 2 * (t % 32) + (wave >> 1));
        copy_from = pool + (size_t)(known(b) ? b : 0) * block_bytes + (wave & 1) * 8 * L::ROW;
        copy_to = ring + at + 8 * wave * L::ROW;
    };
    auto copy_part = [&](int i) {   // i even: of K, odd: of V
        const int key = i / 2 * L::KPC + lane / L::CH, row = 8 * wave + key, c = lane % L::CH;
        if (i & 1) dma16(key * L::ROW + 16 * (c ^ L::vx(row)), copy_from + hkv * head, copy_to + L::HALF + 1024 * (i / 2));
        else dma16(key * L::ROW + 16 * (c ^ L::kx(row)), copy_from, copy_to + 1024 * (i / 2));
    };
    auto copy = [&](int t, uint32_t at) {
        copy_begin(t, at);
#pragma unroll
        for (int i = 0; i < 2 * L::COPIES; ++i) copy_part(i);
    };
#pragma unroll
    for (int i = 0; i < S - 1; ++i)
        if (i < n_tiles) copy(i, i * L::BYTES);

    // the wavefront's columns and the rows that they have: positions w_first .. w_last
    const int c0 = 32 * wave, r0 = bq >= 32 ? c0 & (bq - 1) : 0;
    const int w_rows = min(bq >= 32 ? 32 : bq, rows - r0), w_first = first + r0, w_last = w_first + w_rows - 1;
    bf16x8_t q[TERMS][KK];
    f32x16_t o[NB];
    const int r = c0 + col, t = r & (bq - 1);
    const int pos = t < rows ? first + t : -1;
    float m = -INFINITY, l = 0.f;
    const size_t q_at = (size_t)(seq.first + t0 + min(t, rows - 1)) * a.q_ld + (size_t)((g << pl.log_g) + (r >> log_bq)) * D + 8 * half;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
        float v[8];
        load4(a.q, q_at + 16 * kk, TYPE, v);
        load4(a.q, q_at + 16 * kk + 4, TYPE, v + 4);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            __bf16 s[TERMS];
            split_terms<TERMS>(a.scale < 0.f ? -v[j] : v[j], s);   // (its scores' maximum is then the largest)
#pragma unroll
            for (int i = 0; i < TERMS; ++i) q[i][kk][j] = s[i];
        }
    }
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[b][i] = 0.f;
    bool odd = false;
    const float scale = fabsf(a.scale) * kLog2e;   // scores in base 2
    const uint32_t k_at = ring + col * L::ROW + 16 * (half ^ L::kx(col));   // chunk 2 kk + half of key col, permuted
    const int vk = 4 * half + (lane & 15) / 4;
    const uint32_t v_at = ring + L::HALF + vk * L::ROW + 8 * (lane & 1) + 16 * ((((lane >> 4) & 1) * 2 + (lane & 3) / 2) ^ L::vx(vk));
    const Turns clear = rb.whole(a, first, first + rows - 1), my_clear = rb.whole(a, w_first, max(w_first, w_last));
    Turns mine = widened(rb.touched(a, w_first, max(w_first, w_last)));   // what the wavefront takes part in
    if (w_rows <= 0) mine = Turns{0, 0, 0};
    // This wavefront's share of tile t has landed; with the barrier behind it, everybody's.  In a tile that not every
    // row sees, a V that is not finite must not meet the matrix instructions (0 x inf): it becomes 0 here, and the
    // columns that see it are taken again at the end.
    auto landed = [&](int t, uint32_t at, int behind) {   // behind: tiles under way behind it
        if (S > 5 && behind >= 2) wait_vm<(S > 5 ? 2 : 1) * 2 * L::COPIES>();
        else if (S > 4 && behind >= 1) wait_vm<2 * L::COPIES>();
        else wait_vm<0>();
        asm volatile("" ::: "memory");
        if ((t < n_tiles) & (!clear.has(t) | strange)) {
            at += ring + L::HALF + 8 * wave * L::ROW + 16 * lane;
#pragma unroll
            for (int i = 0; i < L::COPIES; ++i) {
                u32x4 v = *(lds16)(at + 1024 * i);
                const bool bad = clear_odd(v);
                odd |= bad & rb.sees(a, rb.tile_at(t) * KT + 8 * wave + lane / L::CH + L::KPC * i);
                if (bad) *(lds16)(at + 1024 * i) = v;
            }
        }
    };
    auto hide = [&](f32x16_t &s, int t) {
        const int k0 = rb.tile_at(t) * KT + 4 * half;   // the lane's first key; its others are 8 (i / 4) + i % 4 further
        uint32_t pages = t < n_tiles ? ~0u : 0u;
        if (strange && t < n_tiles)
            pages = (known(seq.table[rb.page_at(t, 0)]) ? 0xFFFFu : 0u) | (known(seq.table[rb.page_at(t, 1)]) ? 0xFFFF0000u : 0u);
        hide_scores(s, pages >> (4 * half) & seen_bits(a, pos, k0));
    };
    auto value_frag = [&](uint32_t v, int h, int b) {
        const uint32_t at = (v ^ (64 * b)) + 16 * h * L::ROW;
        const s16x4_t v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds8)at);
        const s16x4_t v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds8)(at + 8 * L::ROW));
        return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    // The maximum that scores are taken relative to: a whole number (so that rescaling is exact, what is already
    // rounded to bf16 included) which stays until a score is 2^kSlack beyond it: p and its sums are floating
    // point, and the rescaling, a quarter of a tile's vector work, is rare after the first tile.
    auto raise = [&](float top, bf16x8_t(&p)[PT][2]) {
        const float best = fmaxf(top, lane_xor(top, 32)) * scale;
        if (__builtin_amdgcn_ballot_w64(best > m + kSlack) == 0) return;
        const float to = best > m + kSlack ? ceilf(best) : m;
        const float alpha = __builtin_amdgcn_exp2f(m - (to == -INFINITY ? 0.f : to));
        m = to;
        l *= alpha;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[b][i] *= alpha;
#pragma unroll
        for (int i = 0; i < PT; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < 8; ++j) p[i][h][j] = (__bf16)((float)p[i][h][j] * alpha);
    };

    f32x16_t s;               // scores of tile t
    bf16x8_t p[PT][2];        // probabilities of tile t - 1
#pragma unroll
    for (int i = 0; i < PT; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) p[i][h] = bf16x8_t{};
    constexpr int N1 = TERMS * KK, N2 = PT * 2 * NB;      // MFMAs of the scores, of the values
    constexpr int EXPS = 8, EXPS1 = EXPS * (N1 + N1 / 8) / (N1 + N2);   // pieces of the softmax (two scores each): behind the scores

    bf16x8_t kf[KK];   // of tile t + 1
    auto load_key = [&](uint32_t at, int kk) { kf[kk] = __builtin_bit_cast(bf16x8_t, *(lds16)((k_at + at) ^ (32 * kk))); };
    auto load_keys = [&](uint32_t at) {
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) load_key(at, kk);
    };
    // tiles 0 and 1 of the S - 1 under way
    landed(0, 0, min(n_tiles, S - 1) - 2);
    landed(1, L::BYTES, min(n_tiles, S - 1) - 2);
    wait_lgkm<0>();
    lds_barrier();
    load_keys(0);
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
#pragma unroll
        for (int i = 0; i < TERMS; ++i) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[kk], q[i][kk], s, 0, 0, 0);
    load_keys(L::BYTES);
    hide(s, 0);
    {
        float top = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
        raise(top, p);
    }
    uint32_t at_new = (S - 1) * L::BYTES, at_keys = 2 * L::BYTES, at_values = 0;   // stages of tiles t + S - 1, t + 2, t - 1
    auto step = [&](uint32_t &at) { at = at == (S - 1) * L::BYTES ? 0 : at + L::BYTES; };
    // The middle of turn t: tile t + 2 has landed everywhere, and tile t - 1 has been read by all: its stage takes
    // tile t + S - 1 (tile S - 1 itself goes to the last stage, which is empty).  The copies are then laid between
    // the values' MFMAs: all wavefronts' at once, behind the barrier, take 580 cycles of a turn of 2200 to issue.
    uint32_t keys_now = 0;
    auto middle = [&](int t) {
        landed(t + 2, at_keys, min(n_tiles, t + S - 1) - (t + 3));
        wait_lgkm<0>();
        lds_barrier();
        if (t + S - 1 < n_tiles) copy_begin(t + S - 1, at_new);
        keys_now = at_keys;
        step(at_new);
        step(at_keys);
        if (t > 0) step(at_values);
    };
    // (on a cache line: where it fell by chance, code in front of it moved the loop's time by up to 3%)
    asm volatile(".p2align 6");
    for (int t = 0; t <= n_tiles; ++t) {   // (turn n_tiles: the last tile's values)
        if (!mine.has(t)) {                // (p is 0 then, and s -inf)
            middle(t);
            load_keys(keys_now);
            if (t + S - 1 < n_tiles) {
#pragma unroll
                for (int i = 0; i < 2 * L::COPIES; ++i) copy_part(i);
            }
            continue;
        }
        f32x16_t n;
        u32x4 pn[PT][2];
        bf16x8_t vf[2 * NB];
        const float ref = m == -INFINITY ? 0.f : m;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) n[i] = 0.f;
        auto softmax_piece = [&](int e) {   // scores 2 e and the one behind it
            const float w0 = __builtin_amdgcn_exp2f(fmaf(s[2 * e], scale, -ref)), w1 = __builtin_amdgcn_exp2f(fmaf(s[2 * e + 1], scale, -ref));
            sum += w0;
            sum += w1;
            uint32_t w[PT];
            split_terms2<PT>(w0, w1, w);
#pragma unroll
            for (int j = 0; j < PT; ++j) pn[j][e / 4][e % 4] = w[j];
            asm volatile("" : "+v"(sum));   // (here, and not where the sums are needed)
        };
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int c = 0; c < N1; ++c) {
            const int kk = c / TERMS, i = c % TERMS;
            n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[kk], q[i][kk], n, 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int f = 0; f < 2 * NB; ++f)
                if (f * N1 / (2 * NB) / 2 == c) vf[f] = value_frag(v_at + at_values, f / NB, f % NB);
#pragma unroll
            for (int e = 0; e < EXPS1; ++e)
                if (e * N1 / EXPS1 == c) softmax_piece(e);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (t == 0) {   // no tile before
#pragma unroll
            for (int f = 0; f < 2 * NB; ++f) vf[f] = bf16x8_t{};
        }
        middle(t);
        const bool more = t + S - 1 < n_tiles;
        if (!my_clear.has(t + 1) | strange) hide(n, t + 1);
        float top;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int c = 0; c < N2; ++c) {
            const int f = c % (2 * NB), i = PT - 1 - c / (2 * NB);   // small terms first; fragment (h, b) = (f / NB, f % NB)
            o[f % NB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[f], p[i][f / NB], o[f % NB], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int e = 0; e < 2 * L::COPIES; ++e)
                if (e * N2 / (2 * L::COPIES) == c && more) copy_part(e);
#pragma unroll
            for (int kk = 0; kk < KK; ++kk)
                if (kk * N2 / KK == c) load_key(keys_now, kk);
#pragma unroll
            for (int e = EXPS1; e < EXPS; ++e)
                if ((e - EXPS1) * N2 / (EXPS - EXPS1) == c) softmax_piece(e);
#pragma unroll
            for (int e = 0; e < EXPS; ++e)
                if (e * N2 / EXPS == c) {
                    const float u = n[2 * e], v = n[2 * e + 1];
                    if (e == 0) top = fmaxf(u, v);
                    else asm("v_max3_f32 %0, %0, %1, %2" : "+v"(top) : "v"(u), "v"(v));   // (fmaxf quiets each operand first)
                }
            __builtin_amdgcn_sched_barrier(0);
        }
        l += sum;
        s = n;
#pragma unroll
        for (int i = 0; i < PT; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) p[i][h] = __builtin_bit_cast(bf16x8_t, pn[i][h]);
        raise(top, p);
    }
    int *const flags = reinterpret_cast<int *>(lds);
    auto store = [&] {
        // Rows are stored 16 bytes a lane, neighbouring lanes side by side, by way of the ring (8 bytes a lane, each row's
        // over 16 instructions: 30 us more of 320 at 4 x 2048 rows of 64 heads).
        constexpr int E = TYPE == STAGE_F32 ? 4 : 2, OROW = D * E + 16, OCH = D * E / 16;
        static_assert(64 + 4 * 32 * OROW <= S * L::BYTES, "the ring holds the output rows");
        char *const out_lds = lds + 64 + wave * 32 * OROW;   // (behind the flags)
        const int out_type = TYPE == STAGE_F32 && seq.first + t0 + t < a.pair_rows ? kPair : TYPE;
        const float sum = l + lane_xor(l, 32);
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                store4(out_lds + col * OROW, 32 * b + 8 * j + 4 * half, out_type,
                       quotient(make_float4(o[b][4 * j], o[b][4 * j + 1], o[b][4 * j + 2], o[b][4 * j + 3]), sum));
#pragma unroll
        for (int i = 0; i < 32 * OCH / 64; ++i) {
            const int e = 64 * i + lane, r = c0 + e / OCH, t = r & (bq - 1);
            const u32x4 v = *reinterpret_cast<const u32x4 *>(out_lds + e / OCH * OROW + e % OCH * 16);
            if (t < rows)
                *reinterpret_cast<u32x4 *>(static_cast<char *>(a.out) + E * ((size_t)(seq.first + t0 + t) * a.out_ld +
                                           (size_t)((g << pl.log_g) + (r >> log_bq)) * D) + e % OCH * 16) = v;
        }
    };
    // Columns that see a V that was cleared, or whose sums are not finite, are taken again; the others keep what they
    // have.  (Rows are stored before, unless out is q, which is read again.)
    const bool same = a.out == a.q;
    __syncthreads();
    if (!same) store();
    const bool bad = t < rows && not_finite(l, o);
    if (lane == 0) flags[wave] = 0;
    if (bad) flags[wave] = 1;
    if (odd) flags[wave] = 2;
    __syncthreads();
    const int any = max(max(flags[0], flags[1]), max(flags[2], flags[3]));
    if (__builtin_expect(any, 0)) by_keys<D, TYPE, STAGE_BF16>(a, rb, g, q_at, pos, bad, any > 1, o, l);
    if (__builtin_expect(any | same, 0)) store();
}

template <int D, int TERMS>
hipError_t launch_tiles(const WindowArgs &a, hipStream_t st) {
    TilePlan p{};
    while (a.n_kv_heads << p.log_g < a.n_q_heads) ++p.log_g;
    // row blocks: no sequence adds more than one that is not full
    const int bq = 128 >> p.log_g, seqs = a.rows.n_seqs < a.rows.rows ? a.rows.n_seqs : a.rows.rows;
    const long blocks = ((long)a.rows.rows / bq + seqs) * a.n_kv_heads;
    if (blocks > kMaxBlocks) return hipErrorInvalidValue;
    STG_LAUNCH((window_tiles<D, TERMS>), dim3((unsigned)blocks), dim3(256), 0, st, a, p);
    return hipGetLastError();
}

// Whether a call's rows go 128 columns to a workgroup (each of which walks all keys that they see) or 16, the keys cut: the
// one that takes less time for the longest list, in us.  Tiles: 8, and for each round of workgroups over the compute units 1 and
// `tile` for 32 keys.  Split: 12, 5 (2) for each round that it could fill, `keys` for 32 keys of a workgroup, shared by all units,
// and 0.1 for 32 keys at all.  (Measured: 245 shapes of 1 to 32 sequences of 17 to 1500 rows, 2 to 40 KV heads, lists of up to
// 5500 keys, types as below.  The kernel taken is 0.5% above the better on the mean, at most 1.31 times; by counts of blocks
// alone it was 10%, up to 3.6 times.)  64 heads of 8 groups, bf16, tiles and split: 1 sequence of 64 rows 9 and 23 us, behind
// 4000 tokens 147 and 77, 16 of 17 rows behind them 177 and 318.
bool by_tiles(const WindowArgs &a) {
    if (a.rows.max_rows * (long)(a.n_q_heads / a.n_kv_heads) <= 16) return false;
    const bool f32 = a.kv_type == STAGE_F32, exact = a.type == STAGE_F32, wide = a.head_dim == 128;
    const double tile = (f32 ? exact ? 2.4 : 1.75 : exact ? 1.3 : 0.9) * (wide ? 1. : 0.67);
    const double keys = f32 ? wide ? 0.9 : 0.57 : wide ? 0.45 : 0.2, round = f32 || wide ? 5. : 2.;
    const long units = device_compute_units(), small = row_blocks(a, 16), large = row_blocks(a, 128);
    auto list = [&](long columns) {   // in tiles
        const long bq = columns * a.n_kv_heads / a.n_q_heads, all = (a.rows.max_len + kTileKeys - 1) / kTileKeys;
        const long listed = (a.sinks + kTileKeys - 1) / kTileKeys + ((long)a.window + bq + 2 * kTileKeys - 3) / kTileKeys;
        return (double)(listed < all ? listed : all);
    };
    const double tiles = 8 + (double)((large + units - 1) / units) * (1 + tile * list(128));
    const double split = 12 + (double)((small + units - 1) / units) * round + list(16) * (keys * (double)small / (double)units + 0.1);
    return tiles < split;
}

}  // namespace

size_t window_workspace(const WindowArgs &a) {
    if (a.rows.rows <= 0 || by_tiles(a)) return 0;
    const SplitPlan p = split_plan(a);
    return p.splits == 1 ? 0 : (size_t)a.rows.rows * a.n_q_heads * p.splits * (a.head_dim + 2) * sizeof(float);
}

hipError_t launch_window_attention(const WindowArgs &a, hipStream_t st) {
    if (a.rows.rows <= 0) return hipSuccess;
    const bool f32 = a.kv_type == STAGE_F32, exact = a.type == STAGE_F32;
    if (f32 && by_tiles(a)) return launch_window_f32(a, st);
#define STG_WINDOW_CASE(D)                                                 \
    if (a.head_dim == D && by_tiles(a))                                    \
        return exact ? launch_tiles<D, 3>(a, st) : launch_tiles<D, 1>(a, st); \
    if (a.head_dim == D)                                                   \
        return f32 ? launch_split<D, true, 1>(a, st)                       \
                   : exact ? launch_split<D, false, 3>(a, st) : launch_split<D, false, 1>(a, st);
    STG_WINDOW_CASE(64) STG_WINDOW_CASE(128)
#undef STG_WINDOW_CASE
    return hipErrorInvalidValue;
}

}  // namespace stg
