// kt_eight.cuh -- eight elements of a row, fp32 or bf16, as fp32 values and back: neighbours, in 16-byte pieces where the
// row allows it (WHOLE: address and first column do), else one by one, those before `cols` only.
// SPREAD (without WHOLE): where each place of a row may hold any column as long as all passes agree, the eight of a thread are 32
// apart, so that a warp's accesses are to neighbours (16384 rows of 1111 bf16 looked up: 47 -> 21 us).
#pragma once

#include <cuda_bf16.h>

#include <cstdint>
#include <cstring>

namespace {

// The column of the e-th of the eight that begin at place c, a multiple of eight.
template <bool SPREAD>
__device__ __forceinline__ int64_t column_of(int64_t c, int e) { return SPREAD ? (c & ~static_cast<int64_t>(255)) + ((c >> 3) & 31) + 32 * e : c + e; }

// The eight as they come from memory, which take the registers of their type only.
template <typename T, bool WHOLE, bool SPREAD = false>
struct Raw {
    uint4 v[sizeof(T) / 2];
    __device__ __forceinline__ void read(const T *row, int64_t c, int64_t cols) {
        if (WHOLE && !SPREAD && c + 8 <= cols) {
#pragma unroll
            for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) v[i] = reinterpret_cast<const uint4 *>(row + c)[i];
        } else {
            T e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int64_t at = column_of<SPREAD>(c, i);
                e[i] = at < cols ? row[at] : T(0.0f);
            }
            memcpy(v, e, sizeof(e));
        }
    }
    __device__ __forceinline__ void get(float (&x)[8]) const {
        const uint32_t *const w = reinterpret_cast<const uint32_t *>(v);
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(w[i] << 16), x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(w[i]);
        }
    }
    __device__ __forceinline__ void add_to(float (&sum)[8]) const {
        float x[8];
        get(x);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] += x[i];
    }
};

template <typename T, bool WHOLE, bool SPREAD = false>
__device__ __forceinline__ void read_eight(const T *row, int64_t c, int64_t cols, float (&v)[8]) {
    Raw<T, WHOLE, SPREAD> raw;
    raw.read(row, c, cols);
    raw.get(v);
}

template <typename T, bool WHOLE, bool SPREAD = false>
__device__ __forceinline__ void write_eight(T *row, int64_t c, int64_t cols, const float (&v)[8]) {
    if (WHOLE && !SPREAD && c + 8 <= cols) {
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
        for (int i = 0; i < 8; ++i) {
            const int64_t at = column_of<SPREAD>(c, i);
            if (at < cols) {
                if constexpr (sizeof(T) == 2) row[at] = __float2bfloat16_rn(v[i]);
                else row[at] = v[i];
            }
        }
    }
}

}  // namespace
