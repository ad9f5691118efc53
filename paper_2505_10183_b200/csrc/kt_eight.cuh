// kt_eight.cuh -- eight neighbouring elements of a row, fp32 or bf16, as fp32 values and back: in 16-byte pieces where the
// row allows it (WHOLE: address and first column do), else one by one, those before `cols` only.
#pragma once

#include <cuda_bf16.h>

#include <cstdint>

namespace {

template <typename T, bool WHOLE>
__device__ __forceinline__ void read_eight(const T *row, int64_t c, int64_t cols, float (&v)[8]) {
    if (WHOLE && c + 8 <= cols) {
        if constexpr (sizeof(T) == 2) {
            const uint4 u = *reinterpret_cast<const uint4 *>(row + c);
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        } else {
            const float4 a = *reinterpret_cast<const float4 *>(row + c), b = *reinterpret_cast<const float4 *>(row + c + 4);
            v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = c + i < cols ? static_cast<float>(row[c + i]) : 0.0f;
    }
}

template <typename T, bool WHOLE>
__device__ __forceinline__ void write_eight(T *row, int64_t c, int64_t cols, const float (&v)[8]) {
    if (WHOLE && c + 8 <= cols) {
        if constexpr (sizeof(T) == 2) {
            uint4 u;
            uint32_t *const w[4] = {&u.x, &u.y, &u.z, &u.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(*w[i]) : "f"(v[2 * i + 1]), "f"(v[2 * i]));
            *reinterpret_cast<uint4 *>(row + c) = u;
        } else {
            *reinterpret_cast<float4 *>(row + c) = make_float4(v[0], v[1], v[2], v[3]);
            *reinterpret_cast<float4 *>(row + c + 4) = make_float4(v[4], v[5], v[6], v[7]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < cols) {
                if constexpr (sizeof(T) == 2) row[c + i] = __float2bfloat16_rn(v[i]);
                else row[c + i] = v[i];
            }
    }
}

}  // namespace
