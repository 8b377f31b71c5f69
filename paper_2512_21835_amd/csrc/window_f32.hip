// Window attention of prompts over an fp32 cache.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "lds_dma.h"
#include "window_rows.h"

namespace stg {
namespace {

// A workgroup: 128 columns = G heads x BQ = 128 / G consecutive rows of one sequence, one KV head; wavefront w the
// columns 32 w .. 32 w + 31 (column r: head r / BQ, row r % BQ).  K and V come in tiles of 32 keys (two pages): fp32 into
// registers a tile ahead, from there as bf16 planes, K as three, whose sum it is, into one of two LDS stages.  S^T = K Q^T and
// O^T += V^T P^T with 32x32x16 MFMAs, lane l holding keys 8 (i / 4) + 4 (l / 32) + i % 4 of the tile for column l % 32, the
// k order of the operand P^T.
//
// fp32 rows: three terms of q and p against three planes hold all 24 bits of each; of the nine products the six largest are
// taken; the others are at most 2^-24 of the whole, of either sign (terms cut from the bits, always toward zero, would leave
// 2^-21).  bf16 rows: q is its one term, so that scores are as exact; p and V are two
// terms each, rounded, which hold both to 2^-16 of their values, as p of bf16 rows everywhere.
//
// In turn t: K of tile t + 1 by Q, then V of tile t - 1 by P, and between their MFMAs the softmax of tile t, the terms of
// K of tile t + 2 and of V of tile t.  2 x 600 fp32 rows of 40 heads behind 300 tokens, window 256: 108 us, 0.6 PFLOP/s
// issued over whole tiles.  A turn takes 3.2 us, 1.6 of them MFMAs, alone on its SIMD (three terms of q, 96 registers, leave
// no room for a second wavefront), and 400 workgroups are two rounds of 256.  Without the overlap 111 us; 16 columns at a
// time with fp32 MFMAs (window_split) 262 us.  bf16 rows: 85 us (69 with K and V as two cut planes and p as one term).
template <int D, int V_PL>
struct PlaneLds {
    static constexpr int K_PL = 3, ROW = 2 * D, PLANE = kTileKeys * ROW, V = K_PL * PLANE, BYTES = V + V_PL * PLANE;   // K's planes, V's
    static constexpr int CHUNKS = D / 64;   // chunks of 8 elements per thread: key tid / 8, chunks tid % 8 + 8 i
    __device__ static int kx(int key) { return D == 128 ? key & 15 : (key >> 1) & 7; }
    __device__ static int vx(int key) { return D == 128 ? (key & 3) << 2 : (key & 2) << 1; }
};

template <int D, int TERMS>
__global__ __launch_bounds__(256, 1) void window_tiles_f32(WindowArgs a, int log_g) {
    constexpr int PT = p_terms(TERMS), V_PL = PT, KK = D / 16, NB = D / 32;
    using L = PlaneLds<D, V_PL>;
    constexpr int K_PL = L::K_PL, TYPE = TERMS == 1 ? STAGE_BF16 : STAGE_F32;
    __shared__ __align__(1024) char lds[2 * L::BYTES];
    __shared__ int flags[4];
    const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hkv = a.n_kv_heads, g = blockIdx.x % hkv, log_bq = 7 - log_g, bq = 1 << log_bq;
    RowBlock rb;
    if (!rb.find(a, blockIdx.x / hkv, log_bq)) return;
    const OpRows::Seq &seq = rb.seq;
    const int t0 = rb.t0, rows = rb.rows, first = rb.first, n_tiles = rb.n_tiles;
    const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
    const size_t head = (size_t)kPage * D, block_elems = (size_t)2 * hkv * head;
    const float *const pool = static_cast<const float *>(a.pool) + g * head;
    auto known = [&](int b) { return (unsigned)b < (unsigned)a.rows.n_blocks; };
    // block ids of the tiles' pages: 64 (32 tiles) in a register of the wavefront, the next 64 under way
    auto ids_from = [&](int t) { return seq.table[rb.page_at(t + lane / 2, lane & 1)]; };
    int ids = 0, more_ids = 0;
    if (n_tiles > 0) {
        ids = ids_from(0);
        more_ids = ids_from(32);
    }
    bool strange = __builtin_amdgcn_ballot_w64(!known(ids)) != 0;   // some page so far is not of the pool

    // The thread's part of a tile: key 8 wave + lane / 8, chunks lane % 8 + 8 i of K and of V.
    f32x4_t raw_k[L::CHUNKS][2], raw_v[L::CHUNKS][2];
    int block_k[2] = {0, 0};   // of the last two tiles whose K was fetched: V's turn comes two tiles later
    auto fetch = [&](f32x4_t(&raw)[L::CHUNKS][2], int b, size_t of) {
        const float *from = pool + (size_t)(known(b) ? b : 0) * block_elems + of + ((wave & 1) * 8 + lane / 8) * D + lane % 8 * 8;
#pragma unroll
        for (int i = 0; i < L::CHUNKS; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) raw[i][h] = *reinterpret_cast<const f32x4_t *>(from + 64 * i + 4 * h);
    };
    auto fetch_k = [&](int t) {   // (t ascending, each once)
        block_k[0] = block_k[1];
        if (t >= n_tiles) return;
        if (t > 0 && t % 32 == 0) {
            ids = more_ids;
            strange |= __builtin_amdgcn_ballot_w64(!known(ids)) != 0;
            more_ids = ids_from(t + 32);
        }
        block_k[1] = __builtin_amdgcn_readlane(ids, 2 * (t % 32) + (wave >> 1));
        fetch(raw_k, block_k[1], 0);
    };
    // A K or V that is not finite (or too large to be rounded to bf16) becomes 0: the columns that see it, if any does, are taken again at the end.
    bool odd = false, bad_k = false, bad_v = false;
    const int my_key = 8 * wave + lane / 8;
    const uint32_t k_to = base + my_key * L::ROW + 16 * (lane % 8 ^ L::kx(my_key));
    const uint32_t v_to = base + L::V + my_key * L::ROW + 16 * (lane % 8 ^ L::vx(my_key));
    u32x4 planes[K_PL];
    using KPlanes = std::integral_constant<int, K_PL>;
    using VPlanes = std::integral_constant<int, V_PL>;
    constexpr int PIECES = 4 * L::CHUNKS;   // two elements each
    auto convert = [&](auto n, const f32x4_t(&raw)[L::CHUNKS][2], uint32_t to, int piece, bool &any_bad) {
        constexpr int PL = decltype(n)::value;
        const int i = piece / 4, e0 = piece % 4 * 2;
        float x[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            x[e] = raw[i][e0 / 4][e0 % 4 + e];
            const bool bad = !(fabsf(x[e]) <= kMaxBf16);
            any_bad |= bad;
            x[e] = bad ? 0.f : x[e];
        }
        uint32_t w[PL];
        split_terms2<PL>(x[0], x[1], w);
#pragma unroll
        for (int p = 0; p < PL; ++p) planes[p][e0 / 2] = w[p];
        if (e0 == 6) {
#pragma unroll
            for (int p = 0; p < PL; ++p) *(lds16)((to ^ (128 * i)) + p * L::PLANE) = planes[p];
        }
    };

    // Whether the thread's key of tile t was bad, if that is a tile and some row sees the key.
    auto noted = [&](bool &bad, int t) {
        if (__builtin_amdgcn_ballot_w64(bad) == 0) return;
        odd |= bad & (t < n_tiles) & rb.sees(a, rb.tile_at(t) * kTileKeys + my_key);
        bad = false;
    };

    // the wavefront's columns and the rows that they have: positions w_first .. w_last
    const int c0 = 32 * wave, r0 = bq >= 32 ? c0 & (bq - 1) : 0;
    const int w_rows = min(bq >= 32 ? 32 : bq, rows - r0), w_first = first + r0, w_last = w_first + w_rows - 1;
    const int r = c0 + col, row = r & (bq - 1), pos = row < rows ? first + row : -1;
    const size_t at = (size_t)((g << log_g) + (r >> log_bq)) * D + 8 * half;
    const size_t q_at = (size_t)(seq.first + t0 + min(row, rows - 1)) * a.q_ld + at;
    fetch_k(0);
    if (n_tiles > 0) fetch(raw_v, block_k[1], hkv * head);
    bf16x8_t q[TERMS][KK];
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
    f32x16_t o[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[b][i] = 0.f;
    float m = -INFINITY, l = 0.f;
    const float scale = fabsf(a.scale) * kLog2e;   // scores in base 2
    const uint32_t k_at = base + col * L::ROW + 16 * (half ^ L::kx(col));   // chunk 2 kk + half of key col, permuted
    const int vk = 4 * half + (lane & 15) / 4;
    const uint32_t v_at = base + L::V + vk * L::ROW + 8 * (lane & 1) + 16 * ((((lane >> 4) & 1) * 2 + (lane & 3) / 2) ^ L::vx(vk));
    auto value_frag = [&](uint32_t v, int h, int b) {
        const uint32_t from = (v ^ (64 * b)) + 16 * h * L::ROW;
        const s16x4_t v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds8)from);
        const s16x4_t v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds8)(from + 8 * L::ROW));
        return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    const Turns clear = rb.whole(a, w_first, max(w_first, w_last));
    Turns mine = widened(rb.touched(a, w_first, max(w_first, w_last)));   // what the wavefront takes part in
    if (w_rows <= 0) mine = Turns{0, 0, 0};
    auto hide = [&](f32x16_t &x, int t) {
        uint32_t pages = t < n_tiles ? ~0u : 0u;
        if (strange && t < n_tiles)
            pages = (known(seq.table[rb.page_at(t, 0)]) ? 0xFFFFu : 0u) | (known(seq.table[rb.page_at(t, 1)]) ? 0xFFFF0000u : 0u);
        hide_scores(x, pages >> (4 * half) & seen_bits(a, pos, rb.tile_at(t) * kTileKeys + 4 * half));
    };
    bf16x8_t p[PT][2];   // probabilities of tile t - 1
#pragma unroll
    for (int i = 0; i < PT; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) p[i][h] = bf16x8_t{};
    // The maximum: a whole number that stays until a score is 2^kSlack beyond it, so that rescaling is exact, and rare.
    auto raise = [&](float top) {
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
    // Groups of MFMAs of one fragment (small terms first), the fragments read AHEAD groups before theirs.
    constexpr int N = K_PL * KK, M = 2 * V_PL * NB, AHEAD = K_PL;
    auto key_frag = [&](uint32_t stage, int c) {
        return __builtin_bit_cast(bf16x8_t, *(lds16)((k_at + stage + (K_PL - 1 - c % K_PL) * L::PLANE) ^ (32 * (c / K_PL))));
    };
    auto value_of = [&](uint32_t stage, int c) { return value_frag(v_at + stage + (V_PL - 1 - c / NB % V_PL) * L::PLANE, c / NB / V_PL, c % NB); };
    auto key_products = [&](f32x16_t &x, const bf16x8_t &k, int c) {
#pragma unroll
        for (int i = TERMS - 1; i >= 0; --i)
            if (i + K_PL - 1 - c % K_PL < K_PL) x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q[i][c / K_PL], x, 0, 0, 0);
    };

    // K of tiles 0 and 1 to their stages; zeros where turn 0 looks for the V of a tile before
#pragma unroll
    for (int e = 0; e < PIECES; ++e) convert(KPlanes{}, raw_k, k_to, e, bad_k);
    noted(bad_k, 0);
    fetch_k(1);
#pragma unroll
    for (int e = 0; e < PIECES; ++e) convert(KPlanes{}, raw_k, k_to + L::BYTES, e, bad_k);
    noted(bad_k, 1);
#pragma unroll
    for (int i = 0; i < L::CHUNKS; ++i)
#pragma unroll
        for (int c = 0; c < V_PL; ++c) *(lds16)((v_to ^ (128 * i)) + L::BYTES + c * L::PLANE) = u32x4{0, 0, 0, 0};
    fetch_k(2);
    wait_lgkm<0>();
    lds_barrier();
    f32x16_t s;   // scores of tile t
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int c = 0; c < N; ++c) key_products(s, key_frag(0, c), c);
    hide(s, 0);
    {
        float top = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
        raise(top);
    }
    for (int t = 0; t <= n_tiles; ++t) {   // (turn n_tiles: the last tile's values)
        // K of tile t + 1 and V of tile t - 1 are in their stages everywhere, and what is written in this turn has no
        // readers left: K of tile t + 2 takes tile t's place, V of tile t that of tile t - 2.  (Behind the last tile
        // what the registers hold goes where nobody reads.)
        wait_lgkm<0>();
        lds_barrier();
        const uint32_t even = (t & 1) * L::BYTES, odd_stage = L::BYTES - even;   // stages of tiles t and t + 2; of t + 1 and t - 1
        if (!mine.has(t)) {   // (p is 0 then, and s -inf)
#pragma unroll
            for (int e = 0; e < PIECES; ++e) convert(KPlanes{}, raw_k, k_to + even, e, bad_k);
            noted(bad_k, t + 2);
#pragma unroll
            for (int e = 0; e < PIECES; ++e) convert(VPlanes{}, raw_v, v_to + even, e, bad_v);
            noted(bad_v, t);
            if (t + 1 < n_tiles) fetch(raw_v, block_k[0], hkv * head);
            fetch_k(t + 3);
            continue;
        }
        f32x16_t n;   // scores of tile t + 1
        u32x4 pn[PT][2];
        bf16x8_t f[AHEAD];
        const float ref = m == -INFINITY ? 0.f : m;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) n[i] = 0.f;
        auto softmax_piece = [&](int e) {   // scores 2 e and 2 e + 1 of tile t
            const float w0 = __builtin_amdgcn_exp2f(fmaf(s[2 * e], scale, -ref)), w1 = __builtin_amdgcn_exp2f(fmaf(s[2 * e + 1], scale, -ref));
            sum += w0;
            sum += w1;
            uint32_t w[PT];
            split_terms2<PT>(w0, w1, w);
#pragma unroll
            for (int j = 0; j < PT; ++j) pn[j][e / 4][e % 4] = w[j];
            asm volatile("" : "+v"(sum));   // (here, and not where the sums are needed)
        };
#pragma unroll
        for (int c = 0; c < AHEAD; ++c) f[c] = key_frag(odd_stage, c);
#pragma unroll
        for (int c = 0; c < N; ++c) {
            __builtin_amdgcn_sched_barrier(0);
            key_products(n, f[c % AHEAD], c);
            if (c + AHEAD < N) f[c % AHEAD] = key_frag(odd_stage, c + AHEAD);
            else f[c % AHEAD] = value_of(odd_stage, c + AHEAD - N);
#pragma unroll
            for (int e = 0; e < PIECES; ++e)
                if (e * N / PIECES == c) convert(KPlanes{}, raw_k, k_to + even, e, bad_k);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e * N / 4 + 1 == c) softmax_piece(e);
            __builtin_amdgcn_sched_barrier(0);
        }
        noted(bad_k, t + 2);
        const int b_v = block_k[0];
        fetch_k(t + 3);
        if (!clear.has(t + 1) | strange) hide(n, t + 1);
        float top = -INFINITY;
        static_assert(N % AHEAD == 0, "the values' first fragments follow the keys' last");
#pragma unroll
        for (int c = 0; c < M; ++c) {
            const int b = c % NB, h = c / NB / V_PL, pl = V_PL - 1 - c / NB % V_PL;
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = PT - 1; i >= 0; --i)
                if (PT < 3 || i + pl < 3) o[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[c % AHEAD], p[i][h], o[b], 0, 0, 0);
            if (c + AHEAD < M) f[c % AHEAD] = value_of(odd_stage, c + AHEAD);
#pragma unroll
            for (int e = 0; e < PIECES; ++e)
                if (e * M / PIECES == c) convert(VPlanes{}, raw_v, v_to + even, e, bad_v);
#pragma unroll
            for (int e = 4; e < 8; ++e)
                if ((e - 4) * M / 4 + 1 == c) softmax_piece(e);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e * M / 8 == c) top = fmaxf(fmaxf(top, n[2 * e]), n[2 * e + 1]);
            __builtin_amdgcn_sched_barrier(0);
        }
        noted(bad_v, t);
        if (t + 1 < n_tiles) fetch(raw_v, b_v, hkv * head);
        l += sum;
        s = n;
#pragma unroll
        for (int i = 0; i < PT; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) p[i][h] = __builtin_bit_cast(bf16x8_t, pn[i][h]);
        raise(top);
    }
    auto store = [&] {
        const float sum = l + lane_xor(l, 32);
        const int out_type = TYPE == STAGE_F32 && seq.first + t0 + row < a.pair_rows ? kPair : TYPE;
        if (row >= rows) return;
        const size_t to = (size_t)(seq.first + t0 + row) * a.out_ld + at - 8 * half;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                store4(a.out, to + 32 * b + 8 * j + 4 * half, out_type,
                       quotient(make_float4(o[b][4 * j], o[b][4 * j + 1], o[b][4 * j + 2], o[b][4 * j + 3]), sum));
    };
    // Columns that see a K or V that was cleared, or whose sums are not finite, are taken again; the others keep what they
    // have.  (Rows are stored before, unless out is q, which is read again: behind this rare code all stores came 2 to 5 us later.)
    const bool same = a.out == a.q;
    if (!same) store();
    const bool bad = row < rows && not_finite(l, o);
    if (lane == 0) flags[wave] = 0;
    if (bad) flags[wave] = 1;
    if (odd) flags[wave] = 2;
    __syncthreads();
    const int any = max(max(flags[0], flags[1]), max(flags[2], flags[3]));
    if (__builtin_expect(any, 0)) by_keys<D, TYPE, STAGE_F32>(a, rb, g, q_at, pos, bad, any > 1, o, l);
    if (__builtin_expect(any | same, 0)) store();
}

template <int D, int TERMS>
hipError_t launch(const WindowArgs &a, hipStream_t st) {
    int log_g = 0;
    while (a.n_kv_heads << log_g < a.n_q_heads) ++log_g;
    // row blocks: no sequence adds more than one that is not full
    const int bq = 128 >> log_g, seqs = a.rows.n_seqs < a.rows.rows ? a.rows.n_seqs : a.rows.rows;
    const long blocks = ((long)a.rows.rows / bq + seqs) * a.n_kv_heads;
    if (blocks > kMaxBlocks) return hipErrorInvalidValue;
    STG_LAUNCH((window_tiles_f32<D, TERMS>), dim3((unsigned)blocks), dim3(256), 0, st, a, log_g);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_window_f32(const WindowArgs &a, hipStream_t st) {
    const bool exact = a.type == STAGE_F32;
    if (a.head_dim == 64) return exact ? launch<64, 3>(a, st) : launch<64, 1>(a, st);
    if (a.head_dim == 128) return exact ? launch<128, 3>(a, st) : launch<128, 1>(a, st);
    return hipErrorInvalidValue;
}

}  // namespace stg
