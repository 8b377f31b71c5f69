// Grouped-query attention with a sliding window and sinks over the paged cache.
#include "lanes.h"
#include "ops_kernels.h"
#include "stage_ops.h"

namespace stg {
namespace {

__device__ __forceinline__ float load_elem(const void *p, size_t e, int type) {
    if (type == STAGE_F32) return static_cast<const float *>(p)[e];
    return __uint_as_float((uint32_t)static_cast<const uint16_t *>(p)[e] << 16);
}

// One wavefront per (row, query head), lane l the elements l and l + 64 of the head: every key in turn.
template <int D>
__global__ __launch_bounds__(64) void window_row_kernel(WindowArgs a) {
    constexpr int E = D / 64;
    const int row = blockIdx.x, h = blockIdx.y, lane = threadIdx.x;
    const int i = a.rows.seq_of(row);
    if (i >= a.rows.n_seqs) return;
    const OpRows::Seq s = a.rows.seq(i);
    if (row - s.first >= a.rows.max_rows) return;
    const int pos = s.pos0 + row - s.first, g = h / (a.n_q_heads / a.n_kv_heads);
    float q[E], o[E], m = -INFINITY, l = 0.f;
    for (int c = 0; c < E; ++c) {
        q[c] = load_elem(a.q, row * (size_t)a.q_ld + h * D + lane + 64 * c, a.type) * a.scale;
        o[c] = 0.f;
    }
    const int end = min(pos + 1, a.rows.max_len), low = max(0, pos + 1 - a.window);
    for (int key = 0; key < end; ++key) {
        if (key < low && key >= a.sinks) key = low;
        if (key >= end) break;
        const int block = s.table[key / kBlockTokens];
        if ((unsigned)block >= (unsigned)a.rows.n_blocks) continue;
        const size_t e = (((size_t)block * 2 * a.n_kv_heads + g) * kBlockTokens + key % kBlockTokens) * D + lane;
        float p = 0.f;
        for (int c = 0; c < E; ++c) p = fmaf(q[c], load_elem(a.pool, e + 64 * c, a.kv_type), p);
        for (int x = 1; x < 64; x *= 2) p += lane_xor(p, x);
        const float top = fmaxf(m, p), ref = top == -INFINITY ? 0.f : top, r = expf(m - ref), w = expf(p - ref);
        l = l * r + w;
        for (int c = 0; c < E; ++c)
            o[c] = fmaf(w, load_elem(a.pool, e + (size_t)a.n_kv_heads * kBlockTokens * D + 64 * c, a.kv_type), o[c] * r);
        m = top;
    }
    for (int c = 0; c < E; ++c) {
        const float v = l > 0.f || l != l ? o[c] / l : 0.f;
        const size_t e = row * (size_t)a.out_ld + h * D + lane + 64 * c;
        if (a.type == STAGE_F32) static_cast<float *>(a.out)[e] = v;
        else static_cast<uint16_t *>(a.out)[e] = __builtin_bit_cast(uint16_t, (__bf16)v);
    }
}

}  // namespace

size_t window_workspace(const WindowArgs &) { return 0; }

hipError_t launch_window_attention(const WindowArgs &a, hipStream_t st) {
    if (a.rows.rows <= 0) return hipSuccess;
    const dim3 grid(a.rows.rows, a.n_q_heads);
    if (a.head_dim == 64) STG_LAUNCH(window_row_kernel<64>, grid, dim3(64), 0, st, a);
    else if (a.head_dim == 128) STG_LAUNCH(window_row_kernel<128>, grid, dim3(64), 0, st, a);
    else return hipErrorInvalidValue;
    return hipGetLastError();
}

}  // namespace stg
