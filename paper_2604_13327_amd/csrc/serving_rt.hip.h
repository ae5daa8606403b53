// Device-side helpers of the serving operators.
#pragma once
#include "device_rt.hip.h"
#include "serving.h"

namespace etc {

// Reports something a kernel found in device memory and did not use (pinned host memory; the last report stays).  Words 2 and 3 in one
// store, then words 0 and 1, by the first of the lanes that refuse: of refusals at the same time, index and value are one's own.
__device__ __forceinline__ void refuse(int32_t *error, int code, int op, int index, int value)
{
    if (lane_id() != __builtin_amdgcn_readfirstlane(lane_id())) return;
    auto pair = [](int a, int b) { return (uint64_t)(uint32_t)b << 32 | (uint32_t)a; };
    uint64_t *word = reinterpret_cast<uint64_t *>(error);
    __hip_atomic_store(as_global(word + 1), pair(index, value), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
    __hip_atomic_store(as_global(word), pair(code, op), __ATOMIC_RELEASE, __HIP_MEMORY_SCOPE_SYSTEM);
}

// Between LDS writes of a wavefront and reads of other lanes of the same one: the LDS keeps their order, the compiler shall.
__device__ __forceinline__ void in_order() { asm volatile("" ::: "memory"); }

typedef __attribute__((ext_vector_type(2))) float f32x2_t;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
// Two values to bf16, round to nearest even (NaN stays NaN).
__device__ __forceinline__ uint32_t to_bf16x2(float a, float b)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{a, b}), bf16x2_t));
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// Inclusive sum over the lanes of a wavefront: within rows of 16 lanes, then the rows' last lanes to the rows behind them.
__device__ __forceinline__ int wave_scan_i(int v)
{
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);      // row_shr 1, 2, 4, 8
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);      // row_bcast 15 into rows 1 and 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);      // row_bcast 31 into rows 2 and 3
    return v;
}

// Largest over the wavefront, the same value in every lane.
__device__ __forceinline__ float wave_max_f(float v)
{
    v = fmaxf(v, dpp_f32<0xB1>(v));
    v = fmaxf(v, dpp_f32<0x4E>(v));
    v = fmaxf(v, dpp_f32<0x141>(v));
    v = fmaxf(v, dpp_f32<0x140>(v));
    auto row = [&](int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane)); };
    return fmaxf(fmaxf(row(0), row(16)), fmaxf(row(32), row(48)));
}

// Sum of a head whose elements lie in D / 16 neighbouring lanes.
template <int D>
__device__ __forceinline__ float head_sum(float v)
{
    v += dpp_f32<0xB1>(v);
    v += dpp_f32<0x4E>(v);
    if (D == 128) v += dpp_f32<0x141>(v);
    return v;
}

}  // namespace etc
