// Norm of the query and key heads, rotation, and append to the paged cache.
#include "lanes.h"
#include "ops_kernels.h"
#include "part_sum.h"
#include "rows8.h"
#include "stage_ops.h"

namespace stg {
namespace {

__device__ __forceinline__ void load_bf16x8(const uint16_t *p, float v[8]) {
    const bf16x8_t b = *reinterpret_cast<const bf16x8_t *>(p);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (float)b[j];
}

// SP parts of fp32 rows, added; 0: bf16 rows.
template <int SP>
__device__ __forceinline__ void load_row8(const AppendArgs &a, size_t e, float v[8]) {
    if constexpr (SP == 0) {
        load_bf16x8(static_cast<const uint16_t *>(a.qkv) + e, v);
    } else {
        const float *p = static_cast<const float *>(a.qkv) + e;
        const float4 x = part_sum<SP>(p, a.part_stride), y = part_sum<SP>(p + 4, a.part_stride);
        v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
        v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
    }
}

__device__ __forceinline__ void load_f32x8(const float *p, float v[8]) {
    const float4 x = reinterpret_cast<const float4 *>(p)[0], y = reinterpret_cast<const float4 *>(p)[1];
    v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
    v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
}

// A thread takes eight neighbouring pairs (i, i + D / 2) of a head, D / 16 threads a head, which add
// their sums of squares by lane exchanges: each element is read once and kept in registers for norm, turn and store.
// Bound by bytes: 8192 bf16 rows of 64 + 16 heads (337 MB) 67 us, 5.0 TB/s; 957 fp32 rows of 40 + 80 heads (118 MB) 32 us, a
// launch too short to reach that.
template <int SP, int D>
__global__ __launch_bounds__(256) void norm_rope_append_kernel(AppendArgs a) {
    constexpr int HALF = D / 2, TPH = D / 16;
    const int row = blockIdx.x;
    const int hq = a.n_q_heads, hkv = a.n_kv_heads, heads = hq + 2 * hkv;
    const int t = blockIdx.y * 256 + threadIdx.x, j = 8 * (t % TPH);
    const int h = min(t / TPH, heads - 1);
    float x1[8], x2[8];
    const size_t e = (size_t)row * a.qkv_ld + (size_t)h * D + j;
    load_row8<SP>(a, e, x1);
    load_row8<SP>(a, e + HALF, x2);

    const int i = a.rows.seq_of(row);
    if (i >= a.rows.n_seqs) return;   // padding
    const OpRows::Seq s = a.rows.seq(i);
    const int place = row - s.first, pos = s.pos0 + place;
    if ((unsigned)place >= (unsigned)a.rows.max_rows || pos < 0 || pos >= a.rows.max_len) return;
    const int block = s.table[pos / kBlockTokens];
    if ((unsigned)block >= (unsigned)a.rows.n_blocks) return;
    int at[3] = {pos, pos, pos};
    if (a.positions) {
        // (an axis without pairs turns nothing by its position)
        at[0] = a.axis1 > 0 ? a.positions[row] : 0;
        at[1] = a.axis1 < a.axis2 ? a.positions[a.rows.rows + row] : 0;
        at[2] = a.axis2 < HALF ? a.positions[2 * (size_t)a.rows.rows + row] : 0;
    }
    for (int x : at)
        if ((unsigned)x >= (unsigned)a.n_angles) return;

    const uint16_t *gain = h < hq ? a.q_gain : h < hq + hkv ? a.k_gain : nullptr;
    float ss = 0.f;
#pragma unroll
    for (int c = 0; c < 8; ++c) ss = fmaf(x1[c], x1[c], ss);
#pragma unroll
    for (int c = 0; c < 8; ++c) ss = fmaf(x2[c], x2[c], ss);
#pragma unroll
    for (int o = TPH / 2; o >= 1; o >>= 1) ss += lane_xor(ss, o);
    if (t >= heads * TPH) return;
    if (gain) {
        const float scale = 1.f / sqrtf(ss / (float)D + a.eps);
        float g1[8], g2[8];
        load_bf16x8(gain + j, g1);
        load_bf16x8(gain + j + HALF, g2);
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            x1[c] = x1[c] * scale * g1[c];
            x2[c] = x2[c] * scale * g2[c];
        }
    }
    if (h < hq + hkv) {
        float cs[8], sn[8];
        if (j + 8 <= a.axis1 || a.axis1 >= HALF) {   // (all eight pairs on the first axis)
            load_f32x8(a.cos_t + (size_t)at[0] * HALF + j, cs);
            load_f32x8(a.sin_t + (size_t)at[0] * HALF + j, sn);
        } else {
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                const int p = j + c < a.axis1 ? at[0] : j + c < a.axis2 ? at[1] : at[2];
                cs[c] = a.cos_t[(size_t)p * HALF + j + c];
                sn[c] = a.sin_t[(size_t)p * HALF + j + c];
            }
        }
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const float r1 = x1[c] * cs[c] - x2[c] * sn[c], r2 = x1[c] * sn[c] + x2[c] * cs[c];
            x1[c] = r1;
            x2[c] = r2;
        }
    }
    if (h < hq) {
        const size_t o = (size_t)row * a.q_ld + (size_t)h * D + j;
        store8(a.q_out, o, a.q_type, x1);
        store8(a.q_out, o + HALF, a.q_type, x2);
    } else {   // head h - hq of K then V
        const size_t o = (((size_t)block * 2 * hkv + h - hq) * kBlockTokens + pos % kBlockTokens) * D + j;
        store8(a.pool, o, a.kv_type, x1);
        store8(a.pool, o + HALF, a.kv_type, x2);
    }
}

template <int D>
hipError_t launch_d(const AppendArgs &a, hipStream_t st) {
    const int threads = (a.n_q_heads + 2 * a.n_kv_heads) * (D / 16);
    const dim3 grid(a.rows.rows, (threads + 255) / 256);
    switch (a.qkv_type == STAGE_BF16 ? 0 : a.n_part) {
#define STG_APPEND_CASE(SP) \
    case SP: STG_LAUNCH((norm_rope_append_kernel<SP, D>), grid, dim3(256), 0, st, a); break;
        STG_APPEND_CASE(0) STG_APPEND_CASE(1) STG_APPEND_CASE(2) STG_APPEND_CASE(3) STG_APPEND_CASE(4) STG_APPEND_CASE(8)
#undef STG_APPEND_CASE
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_norm_rope_append(const AppendArgs &a, hipStream_t st) {
    if (a.rows.rows <= 0) return hipSuccess;
    return a.head_dim == 64 ? launch_d<64>(a, st) : a.head_dim == 128 ? launch_d<128>(a, st) : hipErrorInvalidValue;
}

}  // namespace stg
