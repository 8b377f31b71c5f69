// Internal interface of the operators of include/stage_ops.h: between their C entry points (ops_api.cpp), the
// stage runtime, which runs the same kernels on its own cache, and the kernels (head_norm.hip, window.hip,
// adapter.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "stage_kernels.h"

namespace stg {

// Lengths of a caller's sequences, and windows, count as this at most (lengths as 0 at least): no sum or difference of theirs overflows.
constexpr int kMaxLength = 1 << 30;

// The rows of a call and the cache places of their sequences: the caller's batch (row_start), or the
// equal rows per sequence of a stage call (rows_per_seq of map, its row metadata).  What a kernel takes from device
// memory is clamped here or checked by it: no value of the caller's leads out of a buffer.
struct OpRows {
    const int *row_start, *length;   // null: a stage call
    const int *table;                // [sequences][max_blocks] (a stage's: [n_seq_slots][max_blocks])
    int n_seqs, max_rows, max_len, max_blocks;
    int rows;                        // rows of the buffers
    int n_blocks;                    // blocks of the pool
    RowMap map;

    struct Seq {
        int first, n, pos0;          // first row, rows, position of the first row
        const int *table;
    };
    __device__ __forceinline__ Seq seq(int i) const {
        if (!row_start)
            return {i * map.rows_per_seq, map.rows_per_seq, map.pos0(i), table + (size_t)map.seq_slot(i) * max_blocks};
        const int b = min(max(row_start[i], 0), rows), e = min(max(row_start[i + 1], b), rows);
        return {b, e - b, min(max(length[i], 0), kMaxLength) - (e - b), table + (size_t)i * max_blocks};
    }
    // The sequence of a row: how many of row_start[1 ..] are not above it.  n_seqs for a row of padding.  One load
    // per lane, so that up to 64 sequences cost one round trip; every lane of the wavefront must be active and
    // have the same row.
    __device__ __forceinline__ int seq_of(int row) const {
        if (!row_start) return row / map.rows_per_seq;
        int n = 0;
        for (int i0 = 1; i0 <= n_seqs; i0 += 64) {
            const int i = i0 + (int)__lane_id();
            const int below = __popcll(__builtin_amdgcn_ballot_w64(i <= n_seqs && row_start[min(i, n_seqs)] <= row));
            n += below;
            if (below < 64) break;
        }
        return n;
    }
};

struct AppendArgs {
    const void *qkv;           // fp32 or bf16; fp32: the sum of n_part parts, `part_stride` floats apart
    int qkv_type, n_part;
    size_t part_stride;
    long qkv_ld;
    void *q_out;
    int q_type;
    long q_ld;
    const uint16_t *q_gain, *k_gain;
    float eps;
    const float *cos_t, *sin_t;
    int n_angles;
    const int *positions;      // null: the row's own position
    int axis1, axis2;          // first pairs of the second and third axis (head_dim / 2: none)
    void *pool;
    int n_q_heads, n_kv_heads, head_dim, kv_type;
    OpRows rows;
};
hipError_t launch_norm_rope_append(const AppendArgs &a, hipStream_t st);

struct WindowArgs {
    const void *q;
    void *out;
    int type;                  // of q and out
    long q_ld, out_ld;
    const void *pool;
    int n_q_heads, n_kv_heads, head_dim, kv_type;
    int window, sinks;         // window > 0
    float scale;
    float *part;               // workspace: states of rows whose keys are cut
    int pair_rows;             // (fp32) rows of `out` below it become the hi/lo pair of a GEMM operand, in the row's own bytes
    OpRows rows;
};
// Bytes of WindowArgs::part that a call takes (it looks at the sizes only).
size_t window_workspace(const WindowArgs &a);
hipError_t launch_window_attention(const WindowArgs &a, hipStream_t st);
hipError_t launch_window_f32(const WindowArgs &a, hipStream_t st);   // its prompts over an fp32 cache

struct AdapterArgs {
    const void *x, *base;
    void *out;
    int type;
    int x_pair;                // x: the hi/lo pair of a GEMM operand (x_ld: of the pair)
    long x_ld, base_ld, out_ld;
    int rows, k, n, n_adapters, max_rank;
    const uint16_t *a, *b;
    const int *ids, *ranks;
    const float *scales;
    float *part;               // workspace: A x
};
size_t adapter_workspace(const AdapterArgs &a);
hipError_t launch_adapter_add(const AdapterArgs &a, hipStream_t st);
// ids[row] = of.id[row / rows_per_seq]
struct SeqAdapters {
    int id[kMaxSeqs];
};
hipError_t launch_adapter_rows(const SeqAdapters &of, int rows, int rows_per_seq, int *ids, hipStream_t st);

}  // namespace stg
