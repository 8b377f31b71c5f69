// Low-rank adapters of many requests beside a shared projection.
#include "lanes.h"
#include "ops_kernels.h"
#include "stage_ops.h"

namespace stg {
namespace {

__device__ __forceinline__ float load_elem(const void *p, size_t e, int type) {
    if (type == STAGE_F32) return static_cast<const float *>(p)[e];
    return __uint_as_float((uint32_t)static_cast<const uint16_t *>(p)[e] << 16);
}

__device__ __forceinline__ int rank_of(const AdapterArgs &a, int id) {
    if ((unsigned)id >= (unsigned)a.n_adapters) return 0;
    return a.ranks ? min(max(a.ranks[id], 0), a.max_rank) : a.max_rank;
}

// part[row][j] = scale (A x)_j: a wavefront per (row, j).
__global__ __launch_bounds__(64) void adapter_down_kernel(AdapterArgs a) {
    const int row = blockIdx.x, j = blockIdx.y, id = a.ids[row];
    if (j >= rank_of(a, id)) return;
    const uint16_t *w = a.a + ((size_t)id * a.max_rank + j) * a.k;
    float s = 0.f;
    for (int k = threadIdx.x; k < a.k; k += 64)
        s = fmaf(load_elem(w, k, STAGE_BF16), load_elem(a.x, row * (size_t)a.x_ld + k, a.type), s);
    for (int x = 1; x < 64; x *= 2) s += lane_xor(s, x);
    if (threadIdx.x == 0) a.part[row * (size_t)a.max_rank + j] = s * (a.scales ? a.scales[id] : 1.f);
}

// out = base + B part: a thread per element.
__global__ __launch_bounds__(256) void adapter_up_kernel(AdapterArgs a) {
    const int row = blockIdx.x, c = blockIdx.y * 256 + threadIdx.x, id = a.ids[row], rank = rank_of(a, id);
    if (c >= a.n) return;
    const size_t w = ((size_t)max(id, 0) * a.n + c) * a.max_rank;
    float s = 0.f;
    for (int j = 0; j < rank; ++j) s = fmaf(load_elem(a.b, w + j, STAGE_BF16), a.part[row * (size_t)a.max_rank + j], s);
    const float v = load_elem(a.base, row * (size_t)a.base_ld + c, a.type) + s;
    const size_t e = row * (size_t)a.out_ld + c;
    if (a.type == STAGE_F32) static_cast<float *>(a.out)[e] = v;
    else static_cast<uint16_t *>(a.out)[e] = __builtin_bit_cast(uint16_t, (__bf16)v);
}

}  // namespace

size_t adapter_workspace(const AdapterArgs &a) { return (size_t)a.rows * a.max_rank * sizeof(float); }

hipError_t launch_adapter_add(const AdapterArgs &a, hipStream_t st) {
    if (a.rows <= 0) return hipSuccess;
    STG_LAUNCH(adapter_down_kernel, dim3(a.rows, a.max_rank), dim3(64), 0, st, a);
    STG_LAUNCH(adapter_up_kernel, dim3(a.rows, (a.n + 255) / 256), dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace stg
