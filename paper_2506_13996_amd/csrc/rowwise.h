// Pieces of the kernels that stream rows (embedding, block norms, gradient norm): 16-byte loads and stores of eight
// values, sums over a wavefront and over a workgroup.
#pragma once
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

namespace alst {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

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

// Eight fp32 values from element `at` of a row, a multiple of 4; the lane's offset stays in 32 bits.
__device__ __forceinline__ Raw8<true> load8(const void* row, uint32_t at) {
    const float4* const from = reinterpret_cast<const float4*>(static_cast<const char*>(row) + (size_t)(at * 4u));
    return {{from[0], from[1]}};
}
__device__ __forceinline__ void store8(void* row, uint32_t at, const float (&v)[8]) {
    float4* const to = reinterpret_cast<float4*>(static_cast<char*>(row) + (size_t)(at * 4u));
    to[0] = make_float4(v[0], v[1], v[2], v[3]);
    to[1] = make_float4(v[4], v[5], v[6], v[7]);
}

// Keeps packed values packed through a loop: the compiler would convert them before it, twice the registers.
__device__ __forceinline__ void stay_packed(Raw8<false>& r) { asm volatile("" : "+v"(r.q.x), "+v"(r.q.y), "+v"(r.q.z), "+v"(r.q.w)); }

__device__ __forceinline__ void stay_packed(Raw8<true>&) {}
// Has the values made here: the compiler would put sums off to the loop's end and keep their terms until then.
__device__ __forceinline__ void made_here(float (&v)[8]) {
    asm volatile("" : "+v"(v[0]), "+v"(v[1]), "+v"(v[2]), "+v"(v[3]), "+v"(v[4]), "+v"(v[5]), "+v"(v[6]), "+v"(v[7]));
}

// A row behind a buffer descriptor (its base has to be the same for a wavefront): lanes behind the row's end read zeros and
// write nothing, and so do all lanes of an absent row or matrix, without a branch.
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
template <bool F32>
struct RowBuffer {
    __amdgpu_buffer_rsrc_t rsrc;
    // row `i` of p [*, H]; there: whether it exists
    __device__ __forceinline__ RowBuffer(const void* p, int64_t i, int H, bool there) {
        const int bytes = H * (F32 ? 4 : 2);
        const bool have = there && p != nullptr;
        void* const base = have ? const_cast<char*>(static_cast<const char*>(p)) + i * bytes : nullptr;
        rsrc = __builtin_amdgcn_make_buffer_rsrc(base, (short)0, have ? bytes : 0, 0x00027000);
    }
    __device__ __forceinline__ Raw8<F32> load(uint32_t at) const {      // eight values from element `at`, a multiple of 8
        Raw8<F32> r;
        if constexpr (F32) {
            r.q[0] = __builtin_bit_cast(float4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, at * 4, 0, 0));
            r.q[1] = __builtin_bit_cast(float4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, at * 4 + 16, 0, 0));
        } else {
            r.q = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, at * 2, 0, 0));
        }
        return r;
    }
    // Rounded once.  STREAMS: of a matrix that no cache will hold (bf16 only: fp32 values of a lane fill half a line an instruction).
    template <bool STREAMS = false>
    __device__ __forceinline__ void store(uint32_t at, const float (&v)[8]) const {
        if constexpr (F32) {
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, make_float4(v[0], v[1], v[2], v[3])), rsrc, at * 4, 0, 0);
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, make_float4(v[4], v[5], v[6], v[7])), rsrc, at * 4 + 16, 0, 0);
        } else {
            bf16x8_t o;
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = (__bf16)v[i];
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, o), rsrc, at * 2, 0, STREAMS ? 2 : 0);      // (2: non-temporal)
        }
    }
};

// Sum over the 64 lanes, the same bits in every lane: four steps inside rows of 16 lanes, then the four rows.
template <int CTRL>
__device__ __forceinline__ float from_lane(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
// over each 16 lanes, in all of them
__device__ __forceinline__ float sum_of_16(float v) {
    v += from_lane<0xb1>(v);       // quad_perm 1 0 3 2
    v += from_lane<0x4e>(v);       // quad_perm 2 3 0 1
    v += from_lane<0x141>(v);      // row_half_mirror
    v += from_lane<0x140>(v);      // row_mirror
    return v;
}
__device__ __forceinline__ float wave_sum(float v) {
    v = sum_of_16(v);
    auto row = [&](int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane)); };
    return (row(0) + row(16)) + (row(32) + row(48));
}
__device__ __forceinline__ double wave_sum(double v) {
    for (int step = 1; step < 64; step <<= 1) v += __shfl_xor(v, step);
    return v;
}

// Whether a result of so many bytes is written past the caches.  Behind them is a memory-side cache of 256 MB, from which the next
// call reads a short result: lookup and the norm that reads its rows, both results written so, 8192 x 4096 (64 MB each) 42.7 -> 45.0
// us, 16384 x 4096 89 -> 84, 32768 x 4096 194 -> 173.
static inline bool streams_out(int64_t bytes) { return bytes >= (int64_t)96 << 20; }

static inline bool aligned_to(const void* p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

}  // namespace alst
