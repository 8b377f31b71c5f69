// Eight elements of a row of fp32 or bf16 (STAGE_F32, STAGE_BF16).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "stage_ops.h"

namespace stg {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

__device__ __forceinline__ void store8(void *p, size_t e, int type, const float v[8]) {
    if (type == STAGE_F32) {
        float4 *f = reinterpret_cast<float4 *>(static_cast<float *>(p) + e);
        f[0] = make_float4(v[0], v[1], v[2], v[3]);
        f[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
        bf16x8_t b;
#pragma unroll
        for (int j = 0; j < 8; ++j) b[j] = (__bf16)v[j];   // nearest even
        *reinterpret_cast<bf16x8_t *>(static_cast<uint16_t *>(p) + e) = b;
    }
}

}  // namespace
}  // namespace stg
