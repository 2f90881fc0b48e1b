// Global gradient norm and clipping over a list of tensors (alst_grads.h).
//
// The list travels in the kernels' arguments, kListed tensors a launch, so that a call copies nothing to the device and
// can be captured.  A tensor's bytes are cut into chunks of 16 KB counted from the 16-byte line that its first element lies
// in; a workgroup of 256 threads takes a chunk at a time with four 16-byte loads a thread in flight, and finds the tensor of
// a chunk by a search of the chunk numbers (scalar: the same for the whole workgroup).  A line that a tensor covers
// in part (its first and last) is read by elements.
//
// Bound by HBM: norm and clipping of 3.9 GB of gradients, read twice and written once, 2.00 ms = 5.8 TB/s.  Scaling by a workgroup a
// chunk, in the order of memory, takes 8 % less than by 2048 workgroups that walk, chunks of 16 KB 5 % less than of 32.
#include <algorithm>

#include "../../include/alst_grads.h"
#include "rowwise.h"

namespace alst {

constexpr int kListed = 64;                  // tensors of a launch (32 bytes each of the kernels' arguments)
constexpr int kChunkLines = 1024;            // 16-byte lines of a chunk
constexpr int kThreads = 256;
constexpr int kLinesEach = kChunkLines / kThreads;
constexpr int kMostParts = 1024;             // workgroups (and partial sums) of a launch that adds up, which walk the chunks
constexpr uint32_t kMostClipGroups = 1u << 22;      // workgroups of a launch that scales, one a chunk up to this many
constexpr int64_t kMostBytes = (int64_t)1 << 45;      // of a call's gradients: chunk numbers stay below 2^31

struct GradList {
    const char* g[kListed];
    char* out[kListed];
    int64_t n[kListed];
    uint32_t first[kListed + 1];             // chunk number of a tensor's first chunk; of [count]: the chunks of the launch
    uint64_t fp32;                           // bit t: tensor t is fp32
    int count;
};

// Tensor of a chunk: the last one whose first chunk is not behind it (a tensor of no elements has no chunk).
__device__ __forceinline__ int tensor_of(const GradList& L, uint32_t chunk) {
    int lo = 0, hi = L.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (L.first[mid] <= chunk) lo = mid;
        else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ double square_sum(const uint4& q, bool f32) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
    double s = 0.0;
    if (f32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const double v = __uint_as_float(w[i]);
            s = fma(v, v, s);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const double lo = __uint_as_float(w[i] << 16), hi = __uint_as_float(w[i] & 0xffff0000u);
            s = fma(lo, lo, s);
            s = fma(hi, hi, s);
        }
    }
    return s;
}

// Sum over the workgroup, in every thread, the same bits whatever its size in the launch: wavefronts in order.
__device__ __forceinline__ double block_sum(double v, double* lds) {
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0.0;
    for (int w = 0; w < kThreads / 64; ++w) s += lds[w];
    return s;
}

// Partial sums of squares, one a workgroup.  Squares and sums in fp64: no gradient of either type over- or underflows, and
// the conversions and fused multiply-adds hide behind the loads.
__global__ __launch_bounds__(kThreads) void grad_squares_kernel(GradList L, double* __restrict__ parts) {
    __shared__ double lds[kThreads / 64];
    double s = 0.0;
    const uint32_t chunks = L.first[L.count];
    for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
        const int t = tensor_of(L, c);
        const bool f32 = L.fp32 >> t & 1;
        const int size = f32 ? 4 : 2;
        const char* const base = L.g[t];
        const int64_t phase = reinterpret_cast<uintptr_t>(base) & 15, end = phase + L.n[t] * size;   // bytes from the first line
        const char* const line0 = base - phase;
        const int64_t at0 = (int64_t)(c - L.first[t]) * kChunkLines * 16;
        if (at0 >= phase && at0 + kChunkLines * 16 <= end) {
            const uint4* p = reinterpret_cast<const uint4*>(line0 + at0) + threadIdx.x;
            uint4 q[kLinesEach];
#pragma unroll
            for (int j = 0; j < kLinesEach; ++j) q[j] = p[j * kThreads];
#pragma unroll
            for (int j = 0; j < kLinesEach; ++j) s += square_sum(q[j], f32);
            continue;
        }
        for (int j = 0; j < kLinesEach; ++j) {
            const int64_t at = at0 + ((int64_t)j * kThreads + threadIdx.x) * 16;
            if (at >= phase && at + 16 <= end) {
                s += square_sum(*reinterpret_cast<const uint4*>(line0 + at), f32);
                continue;
            }
            for (int64_t e = at < phase ? phase : at; e < at + 16 && e < end; e += size) {
                const double v = f32 ? *reinterpret_cast<const float*>(line0 + e)
                                     : __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(line0 + e) << 16);
                s = fma(v, v, s);
            }
        }
    }
    s = block_sum(s, lds);
    if (threadIdx.x == 0) parts[blockIdx.x] = s;
}

// The one order in which partial sums are added up.
__device__ __forceinline__ double sum_parts(const double* __restrict__ parts, int n, double* lds) {
    double s = 0.0;
    for (int i = threadIdx.x; i < n; i += kThreads) s += parts[i];
    return block_sum(s, lds);
}

__global__ __launch_bounds__(kThreads) void grad_norm_kernel(const double* __restrict__ parts, int n, double* __restrict__ sumsq,
                                                             float* __restrict__ norm) {
    __shared__ double lds[kThreads / 64];
    const double s = sum_parts(parts, n, lds);
    if (threadIdx.x == 0) {
        if (sumsq) *sumsq = s;
        if (norm) *norm = (float)sqrt(s);
    }
}

// The factor min(1, max_norm / norm) as c * 2^e.  e is 0 unless the factor is below the normal numbers of fp32, where few or none of
// its bits would be left; v * c stays finite, as |v| <= norm < 2^128 and so |v * c| <= norm * factor * 2^-e < 2^127.
// e by two comparisons: 7 tensors of 3.3 MB 9.8 us, with frexp of the factor 10.9.
struct Factor {
    float c;
    int e;
    __device__ __forceinline__ float times(float v) const { return __builtin_ldexpf(v * c, e); }
};
__device__ __forceinline__ Factor factor_of(double ratio) {
    const bool low = ratio < 0x1p-126, very = ratio < 0x1p-251;
    return {(float)(ratio * (very ? 0x1p250 : low ? 0x1p125 : 1.0)), very ? -250 : low ? -125 : 0};
}

__device__ __forceinline__ uint4 scaled(uint4 q, const Factor& c, bool f32) {
    uint32_t* const w = &q.x;
    if (f32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(c.times(__uint_as_float(w[i])));
    } else {
        bf16x8_t o;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            o[2 * i] = (__bf16)c.times(__uint_as_float(w[i] << 16));
            o[2 * i + 1] = (__bf16)c.times(__uint_as_float(w[i] & 0xffff0000u));
        }
        q = __builtin_bit_cast(uint4, o);
    }
    return q;
}

// out = g * c.  Every workgroup adds the partial sums up by itself (n = 1: the sum is there), which pays while there are few
// workgroups: one launch fewer.  The first one writes them down.
template <bool STREAMS>
__global__ __launch_bounds__(kThreads) void grad_clip_kernel(GradList L, const double* __restrict__ parts, int n, float max_norm,
                                                             double* __restrict__ sumsq_out, float* __restrict__ norm_out) {
    __shared__ double lds[kThreads / 64];
    const double sumsq = sum_parts(parts, n, lds), norm = sqrt(sumsq);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        if (sumsq_out) *sumsq_out = sumsq;
        if (norm_out) *norm_out = (float)norm;
    }
    // (a norm that is not finite, in fp32 as it is reported, scales nothing)
    const bool clip = norm > (double)max_norm && isfinite((float)norm);
    const Factor c = factor_of(clip ? (double)max_norm / norm : 1.0);
    const uint32_t chunks = L.first[L.count];
    for (uint32_t k = blockIdx.x; k < chunks; k += gridDim.x) {
        const int t = tensor_of(L, k);
        const bool f32 = L.fp32 >> t & 1;
        const int size = f32 ? 4 : 2;
        const char* const base = L.g[t];
        char* const to = L.out[t];
        if (!clip && base == to) continue;
        const int64_t phase = reinterpret_cast<uintptr_t>(base) & 15, end = phase + L.n[t] * size;
        const char* const line0 = base - phase;
        char* const out0 = to - phase;
        const bool lines = ((reinterpret_cast<uintptr_t>(to) ^ reinterpret_cast<uintptr_t>(base)) & 15) == 0;
        const int64_t at0 = (int64_t)(k - L.first[t]) * kChunkLines * 16;
        if (lines && at0 >= phase && at0 + kChunkLines * 16 <= end) {
            const uint4* p = reinterpret_cast<const uint4*>(line0 + at0) + threadIdx.x;
            uint4* o = reinterpret_cast<uint4*>(out0 + at0) + threadIdx.x;
            uint4 q[kLinesEach];
#pragma unroll
            for (int j = 0; j < kLinesEach; ++j) q[j] = p[j * kThreads];
#pragma unroll
            for (int j = 0; j < kLinesEach; ++j) {
                const u32x4_t w = __builtin_bit_cast(u32x4_t, clip ? scaled(q[j], c, f32) : q[j]);
                u32x4_t* const at = reinterpret_cast<u32x4_t*>(o + j * kThreads);
                if (STREAMS) __builtin_nontemporal_store(w, at);
                else *at = w;
            }
            continue;
        }
        // a chunk at a tensor's end, or of an output at another 16-byte phase: by elements, neighbours in neighbouring lanes
        const int64_t from = std::max(at0, phase), upto = std::min(at0 + (int64_t)kChunkLines * 16, end);
        for (int64_t e = from + (int64_t)threadIdx.x * size; e < upto; e += kThreads * size) {
            if (f32) {
                const float v = *reinterpret_cast<const float*>(line0 + e);
                *reinterpret_cast<float*>(out0 + e) = clip ? c.times(v) : v;
            } else {
                const uint16_t v = *reinterpret_cast<const uint16_t*>(line0 + e);
                const __bf16 o = (__bf16)c.times(__uint_as_float((uint32_t)v << 16));
                *reinterpret_cast<uint16_t*>(out0 + e) = clip ? __builtin_bit_cast(uint16_t, o) : v;
            }
        }
    }
}

// ---- host ----

// The tensors [at, at + kListed) of a list as a launch's argument; at moves behind them.
static GradList take_listed(const alst_grad_tensor* ts, int64_t count, int64_t& at) {
    GradList L = {};
    uint64_t chunks = 0;
    for (; at < count && L.count < kListed; ++at) {
        const alst_grad_tensor& t = ts[at];
        if (t.n == 0) continue;
        const int64_t bytes = t.n * (t.fp32 ? 4 : 2) + (int64_t)(reinterpret_cast<uintptr_t>(t.grad) & 15);
        const uint64_t here = (uint64_t)(bytes + kChunkLines * 16 - 1) / (kChunkLines * 16);
        L.g[L.count] = static_cast<const char*>(t.grad);
        L.out[L.count] = static_cast<char*>(t.out);
        L.n[L.count] = t.n;
        L.first[L.count] = (uint32_t)chunks;
        if (t.fp32) L.fp32 |= (uint64_t)1 << L.count;
        chunks += here;
        ++L.count;
    }
    L.first[L.count] = (uint32_t)chunks;
    return L;
}

static int grid_of(const GradList& L) { return (int)std::min<uint32_t>(L.first[L.count], kMostParts); }

static int validate_grads(const alst_grad_tensor* ts, int64_t count, bool outs) {
    if (!ts) return ALST_ERR_NULL;
    if (count < 1 || count > (int64_t)1 << 20) return ALST_ERR_SHAPE;
    int64_t bytes = 0;
    for (int64_t i = 0; i < count; ++i) {
        const alst_grad_tensor& t = ts[i];
        if (t.n < 0 || t.n > (int64_t)1 << 40) return ALST_ERR_SHAPE;
        if (t.fp32 < 0 || t.fp32 > 1 || t.reserved != 0) return ALST_ERR_UNSUPPORTED;
        if (t.n == 0) continue;
        if (!t.grad || (outs && !t.out)) return ALST_ERR_NULL;
        const uintptr_t size = t.fp32 ? 4 : 2;
        if (!aligned_to(t.grad, size) || (outs && !aligned_to(t.out, size))) return ALST_ERR_ALIGN;
        bytes += t.n * (int64_t)size;
        if (bytes > kMostBytes) return ALST_ERR_SHAPE;
    }
    return ALST_OK;
}

static int64_t parts_room(int64_t count) { return (count + kListed - 1) / kListed * kMostParts; }

// Partial sums of all launches into `parts`; their number into n.
static int run_squares(const alst_grad_tensor* ts, int64_t count, double* parts, int64_t& n, hipStream_t s) {
    n = 0;
    for (int64_t at = 0; at < count;) {
        const GradList L = take_listed(ts, count, at);
        if (L.count == 0) break;
        const int grid = grid_of(L);
        hipLaunchKernelGGL(grad_squares_kernel, dim3(grid), dim3(kThreads), 0, s, L, parts + n);
        n += grid;
    }
    return hipGetLastError() == hipSuccess ? ALST_OK : ALST_ERR_HIP;
}

static int run_clip(const alst_grad_tensor* ts, int64_t count, const double* parts, int n, float max_norm, double* sumsq_out,
                    float* norm_out, hipStream_t s) {
    int64_t bytes = 0;
    for (int64_t i = 0; i < count; ++i) bytes += ts[i].n * (ts[i].fp32 ? 4 : 2);
    // (the gradients are read a second time, so what is written besides should not take their place in the caches: 355 MB 202 -> 188 us)
    auto kernel = streams_out(bytes) ? grad_clip_kernel<true> : grad_clip_kernel<false>;
    bool first = true;
    for (int64_t at = 0; at < count || first;) {
        const GradList L = take_listed(ts, count, at);
        // (a list of empty tensors still has a norm)
        hipLaunchKernelGGL(kernel, dim3(std::max<uint32_t>(std::min(L.first[L.count], kMostClipGroups), 1)), dim3(kThreads), 0, s, L, parts, n, max_norm,
                           first ? sumsq_out : nullptr, first ? norm_out : nullptr);
        first = false;
    }
    return hipGetLastError() == hipSuccess ? ALST_OK : ALST_ERR_HIP;
}

static int check_workspace(int64_t count, const void* ws, size_t bytes) {
    if (!ws) return ALST_ERR_NULL;
    if (!aligned_to(ws, 16)) return ALST_ERR_ALIGN;
    return bytes < alst_grad_norm_workspace_bytes(count) ? ALST_ERR_WORKSPACE : ALST_OK;
}

}  // namespace alst

using namespace alst;

extern "C" {

size_t alst_grad_norm_workspace_bytes(int64_t count) {
    if (count < 1 || count > (int64_t)1 << 20) return 0;
    return (size_t)(parts_room(count) + 2) * sizeof(double);
}

int alst_grad_norm(const alst_grad_tensor* tensors, int64_t count, double* sumsq_out, float* norm_out, void* workspace,
                   size_t workspace_bytes, void* stream) {
    int rc = validate_grads(tensors, count, false);
    if (rc == ALST_OK && !sumsq_out) rc = ALST_ERR_NULL;
    if (rc == ALST_OK && (!aligned_to(sumsq_out, 8) || !aligned_to(norm_out, 4))) rc = ALST_ERR_ALIGN;
    if (rc == ALST_OK) rc = check_workspace(count, workspace, workspace_bytes);
    if (rc != ALST_OK) return rc;
    double* const parts = static_cast<double*>(workspace);
    int64_t n;
    rc = run_squares(tensors, count, parts, n, (hipStream_t)stream);
    if (rc != ALST_OK) return rc;
    hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(kThreads), 0, (hipStream_t)stream, parts, (int)n, sumsq_out, norm_out);
    return hipGetLastError() == hipSuccess ? ALST_OK : ALST_ERR_HIP;
}

int alst_grad_clip(const alst_grad_tensor* tensors, int64_t count, const double* sumsq, float max_norm, float* norm_out,
                   void* stream) {
    int rc = validate_grads(tensors, count, true);
    if (rc == ALST_OK && !sumsq) rc = ALST_ERR_NULL;
    if (rc == ALST_OK && (!aligned_to(sumsq, 8) || !aligned_to(norm_out, 4))) rc = ALST_ERR_ALIGN;
    if (rc == ALST_OK && !(max_norm > 0.f)) rc = ALST_ERR_UNSUPPORTED;
    if (rc != ALST_OK) return rc;
    return run_clip(tensors, count, sumsq, 1, max_norm, nullptr, norm_out, (hipStream_t)stream);
}

int alst_grad_norm_clip(const alst_grad_tensor* tensors, int64_t count, float max_norm, double* sumsq_out, float* norm_out,
                        void* workspace, size_t workspace_bytes, void* stream) {
    int rc = validate_grads(tensors, count, true);
    if (rc == ALST_OK && (!aligned_to(sumsq_out, 8) || !aligned_to(norm_out, 4))) rc = ALST_ERR_ALIGN;
    if (rc == ALST_OK && !(max_norm > 0.f)) rc = ALST_ERR_UNSUPPORTED;
    if (rc == ALST_OK) rc = check_workspace(count, workspace, workspace_bytes);
    if (rc != ALST_OK) return rc;
    double* const parts = static_cast<double*>(workspace);
    int64_t n;
    rc = run_squares(tensors, count, parts, n, (hipStream_t)stream);
    if (rc != ALST_OK) return rc;
    // (fewer chunks than workgroups that add up: 7 tensors of 3.3 MB 11.2 us, 14.6 with a launch for the sum)
    if (n < kMostParts)
        return run_clip(tensors, count, parts, (int)n, max_norm, sumsq_out, norm_out, (hipStream_t)stream);
    double* const sum = parts + parts_room(count);
    hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(kThreads), 0, (hipStream_t)stream, parts, (int)n, sum, (float*)nullptr);
    return run_clip(tensors, count, sum, 1, max_norm, sumsq_out, norm_out, (hipStream_t)stream);
}

}  // extern "C"
