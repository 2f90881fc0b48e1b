// Pieces of the kernels that stream rows (embedding, block norms, gradient norm): 16-byte loads and stores of eight
// values, sums over a wavefront and over a workgroup.
#pragma once
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "common.h"

namespace alst {

// Eight values of a row: 16 bytes of bf16, or 32 of fp32, as they were loaded (bf16 stays packed until it is used).
template <bool F32> struct Raw8;
template <> struct Raw8<false> {
    uint4 q;
    __device__ __forceinline__ float get(int i) const {
        const uint32_t w = (&q.x)[i >> 1];
        return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
    }
};
template <> struct Raw8<true> {
    float4 q[2];
    __device__ __forceinline__ float get(int i) const { return (&q[i >> 2].x)[i & 3]; }
};

template <bool F32>
__device__ __forceinline__ Raw8<F32> load8(const void* p, int64_t at) {      // element `at`, a multiple of 8
    Raw8<F32> r;
    if constexpr (F32) {
        const float4* f = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(p) + at);
        r.q[0] = f[0];
        r.q[1] = f[1];
    } else {
        r.q = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(p) + at);
    }
    return r;
}
template <bool F32>
__device__ __forceinline__ Raw8<F32> zero8() {
    Raw8<F32> r;
    if constexpr (F32) r.q[0] = r.q[1] = make_float4(0.f, 0.f, 0.f, 0.f);
    else r.q = make_uint4(0u, 0u, 0u, 0u);
    return r;
}

// Eight fp32 values rounded once to the row's type.
template <bool F32>
__device__ __forceinline__ void store8(void* p, int64_t at, const float (&v)[8]) {
    if constexpr (F32) {
        float4* f = reinterpret_cast<float4*>(reinterpret_cast<float*>(p) + at);
        f[0] = make_float4(v[0], v[1], v[2], v[3]);
        f[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
        bf16x8_t o;
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = (__bf16)v[i];
        *reinterpret_cast<bf16x8_t*>(reinterpret_cast<uint16_t*>(p) + at) = o;
    }
}

// Sum over the 64 lanes, the same bits in every lane: four steps inside rows of 16 lanes, then the four rows.
__device__ __forceinline__ float wave_sum(float v) {
    auto from = [](float x, auto ctrl) {
        return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), decltype(ctrl)::value, 0xf, 0xf, true));
    };
    v += from(v, std::integral_constant<int, 0xb1>{});       // quad_perm 1 0 3 2
    v += from(v, std::integral_constant<int, 0x4e>{});       // quad_perm 2 3 0 1
    v += from(v, std::integral_constant<int, 0x141>{});      // row_half_mirror
    v += from(v, std::integral_constant<int, 0x140>{});      // row_mirror
    auto row = [&](int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane)); };
    return (row(0) + row(16)) + (row(32) + row(48));
}
__device__ __forceinline__ double wave_sum(double v) {
    for (int step = 1; step < 64; step <<= 1) v += __shfl_xor(v, step);
    return v;
}

static inline bool aligned_to(const void* p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

}  // namespace alst
