// The norms around a block with its gate and scaled residual addition (alst_block_norm.h), forward and backward.
//
// A row is held in the registers of W wavefronts, 8 * VPT values a lane, so that everything is read and written once; its
// sums (mean squares, and in backward the two products of a norm's gradient) go over the wavefronts through LDS.  A
// workgroup holds R = max(1, 4 / W) rows at a time and walks the rows of the call.
#include <algorithm>

#include "../../include/alst_block_norm.h"
#include "rowwise.h"

namespace alst {

constexpr int64_t kMaxNormH = 16384;
constexpr int kMaxNormParts = 1024;            // workgroups of a backward launch: rows of partial weight gradients

struct NormParams {
    const void *residual, *d_residual_out;
    const uint16_t *branch, *w_post, *gate, *w_pre, *d_normed;
    void *residual_out, *d_residual;
    uint16_t *normed, *d_branch, *d_gate;
    float* parts;                              // [workgroup][2][H]: dw_pre, dw_post
    int64_t N;
    int H, gate_cols;
    float scale, eps, offset;
};

// A workgroup's place: R rows of W wavefronts.
struct RowPlace {
    int W, R, row, tid;                        // tid: thread of the row
    float* lds;                                // [2][R][W][2]
    int turn;
    __device__ __forceinline__ RowPlace(float* lds_) : W(blockDim.x >> 6), R(blockDim.y), row(threadIdx.y), tid(threadIdx.x), lds(lds_), turn(0) {}
    // Sums of two values over the row.  The room alternates, so a sum's readers are done when its room comes up again.
    __device__ __forceinline__ void sum2(float& a, float& b) {
        a = wave_sum(a);
        b = wave_sum(b);
        if (W == 1) return;
        float* const at = lds + (turn * R + row) * W * 2;
        turn ^= 1;
        if ((tid & 63) == 0) {
            at[(tid >> 6) * 2] = a;
            at[(tid >> 6) * 2 + 1] = b;
        }
        __syncthreads();
        a = b = 0.f;
        for (int w = 0; w < W; ++w) {
            a += at[w * 2];
            b += at[w * 2 + 1];
        }
    }
    __device__ __forceinline__ void sum1(float& a) {
        float none = 0.f;
        sum2(a, none);
    }
};

// sigmoid(z) and 1 - sigmoid(z), both to a few steps of fp32 however large |z| is.
struct Gate { float on, off; };
__device__ __forceinline__ Gate gate_of(float z) {
    const float t = expf(-fabsf(z)), s = 1.f / (1.f + t);
    return z >= 0.f ? Gate{s, t * s} : Gate{t * s, s};
}
__device__ __forceinline__ float bf16_value(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }

template <bool F32, int VPT>
__global__ __launch_bounds__(1024) void norm_forward_kernel(NormParams p) {
    extern __shared__ float lds[];
    RowPlace at(lds);
    const float inv_h = 1.f / p.H;
    int col[VPT];
    bool in[VPT];
    Raw8<false> w1[VPT], w2[VPT];
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
        col[v] = (v * (at.W * 64) + at.tid) * 8;
        in[v] = col[v] < p.H;
        w1[v] = p.w_post && in[v] ? load8<false>(p.w_post, col[v]) : zero8<false>();
        w2[v] = p.w_pre && in[v] ? load8<false>(p.w_pre, col[v]) : zero8<false>();
    }
    for (int64_t i0 = (int64_t)blockIdx.x * at.R; i0 < p.N; i0 += (int64_t)gridDim.x * at.R) {
        const int64_t i = i0 + at.row, base = i * p.H;
        const bool row_in = i < p.N;
        Raw8<F32> r[VPT];
        Raw8<false> b[VPT], z[VPT];
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            const bool here = row_in && in[v];
            r[v] = here ? load8<F32>(p.residual, base + col[v]) : zero8<F32>();
            b[v] = here && p.branch ? load8<false>(p.branch, base + col[v]) : zero8<false>();
            z[v] = here && p.gate_cols > 1 ? load8<false>(p.gate, base + col[v]) : zero8<false>();
        }
        float x[VPT][8];
        if (p.branch) {
            float q1 = 1.f;
            if (p.w_post) {
                float bb = 0.f;
#pragma unroll
                for (int v = 0; v < VPT; ++v)
#pragma unroll
                    for (int k = 0; k < 8; ++k) bb += b[v].get(k) * b[v].get(k);
                at.sum1(bb);
                q1 = 1.f / sqrtf(bb * inv_h + p.eps);
            }
            const float s = p.gate_cols == 1 && row_in ? p.scale * gate_of(bf16_value(p.gate + i)).on : p.scale;
#pragma unroll
            for (int v = 0; v < VPT; ++v) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    float change = s * b[v].get(k);
                    if (p.w_post) change *= q1 * (w1[v].get(k) + p.offset);
                    if (p.gate_cols > 1) change *= gate_of(z[v].get(k)).on;
                    x[v][k] = r[v].get(k) + change;
                }
                if (row_in && in[v]) store8<F32>(p.residual_out, base + col[v], x[v]);
            }
        } else {
#pragma unroll
            for (int v = 0; v < VPT; ++v)
#pragma unroll
                for (int k = 0; k < 8; ++k) x[v][k] = r[v].get(k);
        }
        if (p.w_pre) {
            float xx = 0.f;
#pragma unroll
            for (int v = 0; v < VPT; ++v)
#pragma unroll
                for (int k = 0; k < 8; ++k) xx += x[v][k] * x[v][k];
            at.sum1(xx);
            const float q2 = 1.f / sqrtf(xx * inv_h + p.eps);
#pragma unroll
            for (int v = 0; v < VPT; ++v) {
                float n[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) n[k] = x[v][k] * q2 * (w2[v].get(k) + p.offset);
                if (row_in && in[v]) store8<false>(p.normed, base + col[v], n);
            }
        }
    }
}

template <bool F32, int VPT>
__global__ __launch_bounds__(1024) void norm_backward_kernel(NormParams p) {
    extern __shared__ float lds[];
    RowPlace at(lds);
    const float inv_h = 1.f / p.H;
    int col[VPT];
    bool in[VPT];
    Raw8<false> w1[VPT], w2[VPT];
    float dw1[VPT][8], dw2[VPT][8];
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
        col[v] = (v * (at.W * 64) + at.tid) * 8;
        in[v] = col[v] < p.H;
        w1[v] = p.w_post && in[v] ? load8<false>(p.w_post, col[v]) : zero8<false>();
        w2[v] = p.w_pre && in[v] ? load8<false>(p.w_pre, col[v]) : zero8<false>();
#pragma unroll
        for (int k = 0; k < 8; ++k) dw1[v][k] = dw2[v][k] = 0.f;
    }
    const bool post = p.w_post != nullptr, gated = p.gate_cols != 0;
    for (int64_t i0 = (int64_t)blockIdx.x * at.R; i0 < p.N; i0 += (int64_t)gridDim.x * at.R) {
        const int64_t i = i0 + at.row, base = i * p.H;
        const bool row_in = i < p.N;
        Raw8<F32> r[VPT], up[VPT];
        Raw8<false> b[VPT], dn[VPT], z[VPT];
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            const bool here = row_in && in[v];
            r[v] = here && p.w_pre ? load8<F32>(p.residual, base + col[v]) : zero8<F32>();
            dn[v] = here && p.w_pre ? load8<false>(p.d_normed, base + col[v]) : zero8<false>();
            up[v] = here && p.d_residual_out ? load8<F32>(p.d_residual_out, base + col[v]) : zero8<F32>();
            b[v] = here && (post || gated) ? load8<false>(p.branch, base + col[v]) : zero8<false>();
            z[v] = here && p.gate_cols > 1 ? load8<false>(p.gate, base + col[v]) : zero8<false>();
        }
        float bb = 0.f, q1 = 1.f;
        if (post) {
#pragma unroll
            for (int v = 0; v < VPT; ++v)
#pragma unroll
                for (int k = 0; k < 8; ++k) bb += b[v].get(k) * b[v].get(k);
            at.sum1(bb);
            q1 = 1.f / sqrtf(bb * inv_h + p.eps);
        }
        float g[VPT][8];                       // dr
        if (p.w_pre) {
            float rr = 0.f, ur = 0.f;
#pragma unroll
            for (int v = 0; v < VPT; ++v)
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    rr += r[v].get(k) * r[v].get(k);
                    ur += dn[v].get(k) * (w2[v].get(k) + p.offset) * r[v].get(k);
                }
            at.sum2(rr, ur);
            const float q2 = 1.f / sqrtf(rr * inv_h + p.eps), c = q2 * q2 * ur * inv_h;
#pragma unroll
            for (int v = 0; v < VPT; ++v)
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    g[v][k] = up[v].get(k) + q2 * (dn[v].get(k) * (w2[v].get(k) + p.offset) - r[v].get(k) * c);
                    dw2[v][k] += dn[v].get(k) * (r[v].get(k) * q2);
                }
        } else {
#pragma unroll
            for (int v = 0; v < VPT; ++v)
#pragma unroll
                for (int k = 0; k < 8; ++k) g[v][k] = up[v].get(k);
        }
        if (p.d_residual) {
#pragma unroll
            for (int v = 0; v < VPT; ++v)
                if (row_in && in[v]) store8<F32>(p.d_residual, base + col[v], g[v]);
        }
        if (!p.d_branch) continue;
        // dp, in g's place; sum over the row of (dp without a row's gate factor) * (w_post + o) * b: of use to both the norm's and
        // the row gate's gradient
        const Gate row_gate = p.gate_cols == 1 && row_in ? gate_of(bf16_value(p.gate + i)) : Gate{1.f, 0.f};
        const float s = p.scale * row_gate.on;
        float vb = 0.f;
        float off[VPT][8];
#pragma unroll
        for (int v = 0; v < VPT; ++v)
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const Gate gate = p.gate_cols > 1 ? gate_of(z[v].get(k)) : Gate{1.f, 0.f};
                off[v][k] = gate.off;
                g[v][k] *= s * gate.on;
                if (post) dw1[v][k] += g[v][k] * (b[v].get(k) * q1);
                vb += g[v][k] * (post ? w1[v].get(k) + p.offset : 1.f) * b[v].get(k);
            }
        if (post || p.gate_cols == 1) at.sum1(vb);
        if (p.gate_cols == 1 && row_in && at.tid == 0) {
            const __bf16 dz = (__bf16)(row_gate.off * q1 * vb);
            p.d_gate[i] = __builtin_bit_cast(uint16_t, dz);
        }
        const float c = q1 * q1 * vb * inv_h;
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            float o[8], dz[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float w = post ? w1[v].get(k) + p.offset : 1.f;
                if (p.gate_cols > 1) dz[k] = g[v][k] * off[v][k] * (q1 * w * b[v].get(k));
                o[k] = post ? q1 * (g[v][k] * w - b[v].get(k) * c) : g[v][k];
            }
            if (row_in && in[v]) {
                store8<false>(p.d_branch, base + col[v], o);
                if (p.gate_cols > 1) store8<false>(p.d_gate, base + col[v], dz);
            }
        }
    }
    // the rows of the workgroup together, then its partial sums of the weights' gradients
    float* const part = p.parts + (int64_t)blockIdx.x * 2 * p.H;
    for (int which = 0; which < 2; ++which) {
        if (!(which ? post : p.w_pre != nullptr)) continue;
        if (at.R > 1) {
            __syncthreads();
#pragma unroll
            for (int v = 0; v < VPT; ++v)
                if (in[v]) store8<true>(lds, (int64_t)at.row * p.H + col[v], which ? dw1[v] : dw2[v]);
            __syncthreads();
            for (int c = at.row * blockDim.x + at.tid; c < p.H; c += blockDim.x * at.R) {
                float t = 0.f;
                for (int y = 0; y < at.R; ++y) t += lds[y * p.H + c];
                part[(int64_t)which * p.H + c] = t;
            }
        } else {
#pragma unroll
            for (int v = 0; v < VPT; ++v)
                if (in[v]) store8<true>(part, (int64_t)which * p.H + col[v], which ? dw1[v] : dw2[v]);
        }
    }
}

// Weight gradients: the workgroups' partial sums of 64 columns, 16 threads a column.
__global__ __launch_bounds__(1024) void norm_weights_kernel(const float* __restrict__ parts, int n, int H, void* dw_pre, void* dw_post,
                                                            bool f32, bool accumulate) {
    __shared__ float lds[16][64];
    const int lane = threadIdx.x & 63, y = threadIdx.x >> 6, which = blockIdx.y, c = blockIdx.x * 64 + lane;
    void* const out = which ? dw_post : dw_pre;
    if (!out) return;
    float s = 0.f;
    if (c < H)
        for (int k = y; k < n; k += 16) s += parts[((int64_t)k * 2 + which) * H + c];
    lds[y][lane] = s;
    __syncthreads();
    if (y == 0 && c < H) {
        s = 0.f;
        for (int k = 0; k < 16; ++k) s += lds[k][lane];
        if (f32) {
            float* const o = static_cast<float*>(out) + c;
            *o = accumulate ? *o + s : s;
        } else {
            uint16_t* const o = static_cast<uint16_t*>(out) + c;
            const __bf16 r = (__bf16)(accumulate ? bf16_value(o) + s : s);
            *o = __builtin_bit_cast(uint16_t, r);
        }
    }
}

// ---- host ----

struct NormShape { int W, R, vpt; };
static NormShape norm_shape(int64_t H) {
    const int vpt = H <= 512 ? 1 : 2;
    const int W = (int)((H + 512 * vpt - 1) / (512 * vpt));
    return {W, W == 1 ? 4 : W == 2 ? 2 : 1, vpt};
}
static int64_t norm_parts(int64_t N, int64_t H) {
    const NormShape s = norm_shape(H);
    return std::min<int64_t>((N + s.R - 1) / s.R, kMaxNormParts);
}

static bool norm_shape_ok(int64_t N, int64_t H) { return N >= 1 && N <= (int64_t)1 << 30 && H >= 1 && H <= kMaxNormH; }

static int validate_norm(const NormParams& p, int64_t H, int64_t gate_cols) {
    if (!norm_shape_ok(p.N, H)) return ALST_ERR_SHAPE;
    if (p.gate ? gate_cols != 1 && gate_cols != H : gate_cols != 0) return ALST_ERR_SHAPE;
    if (H % 8 != 0) return ALST_ERR_ALIGN;
    const void* ptrs[] = {p.residual, p.d_residual_out, p.branch, p.w_post, p.gate, p.w_pre, p.d_normed, p.residual_out, p.d_residual,
                          p.normed, p.d_branch, p.d_gate, p.parts};
    for (const void* q : ptrs)
        if (!aligned_to(q, 16)) return ALST_ERR_ALIGN;
    if (!(p.eps >= 1.17549435e-38f) || !(p.eps <= 3.402823466e38f)) return ALST_ERR_UNSUPPORTED;
    return ALST_OK;
}

}  // namespace alst

using namespace alst;

extern "C" {

size_t alst_block_norm_workspace_bytes(int64_t N, int64_t H) {
    return norm_shape_ok(N, H) ? (size_t)norm_parts(N, H) * 2 * H * 4 : 0;
}

int alst_block_norm_forward(const void* residual, const void* branch, const void* w_post, const void* gate, int64_t gate_cols,
                            const void* w_pre, int64_t N, int64_t H, float branch_scale, float eps, float weight_offset,
                            void* residual_out, void* normed, uint32_t flags, void* stream) {
    if (!residual) return ALST_ERR_NULL;
    if (!branch ? (!w_pre || w_post || gate || residual_out) : !residual_out) return ALST_ERR_NULL;
    if ((w_pre != nullptr) != (normed != nullptr)) return ALST_ERR_NULL;
    if (flags & ~ALST_FLAG_RESIDUAL_FP32) return ALST_ERR_UNSUPPORTED;
    NormParams p = {};
    p.residual = residual; p.branch = (const uint16_t*)branch; p.w_post = (const uint16_t*)w_post; p.gate = (const uint16_t*)gate;
    p.w_pre = (const uint16_t*)w_pre; p.residual_out = residual_out; p.normed = (uint16_t*)normed;
    p.N = N; p.scale = branch_scale; p.eps = eps; p.offset = weight_offset;
    const int rc = validate_norm(p, H, gate_cols);
    if (rc != ALST_OK) return rc;
    p.H = (int)H; p.gate_cols = (int)gate_cols;
    const NormShape s = norm_shape(H);
    const bool f32 = flags & ALST_FLAG_RESIDUAL_FP32;
    auto kernel = s.vpt == 1 ? (f32 ? norm_forward_kernel<true, 1> : norm_forward_kernel<false, 1>)
                             : (f32 ? norm_forward_kernel<true, 2> : norm_forward_kernel<false, 2>);
    const int64_t grid = std::min<int64_t>((N + s.R - 1) / s.R, 256 * 8);
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(s.W * 64, s.R), 2 * s.R * s.W * 2 * sizeof(float), (hipStream_t)stream, p);
    return hipGetLastError() == hipSuccess ? ALST_OK : ALST_ERR_HIP;
}

int alst_block_norm_backward(const void* residual_out, const void* branch, const void* w_post, const void* gate, int64_t gate_cols,
                             const void* w_pre, const void* d_normed, const void* d_residual_out, int64_t N, int64_t H,
                             float branch_scale, float eps, float weight_offset, void* d_residual, void* d_branch, void* d_gate,
                             void* dw_post, void* dw_pre, void* workspace, size_t workspace_bytes, uint32_t flags, void* stream) {
    if (w_pre ? !residual_out || !d_normed || !dw_pre || !d_residual : d_normed || dw_pre || !d_residual_out) return ALST_ERR_NULL;
    if ((w_post != nullptr) != (dw_post != nullptr) || (gate != nullptr) != (d_gate != nullptr)) return ALST_ERR_NULL;
    if ((w_post || gate) && !branch) return ALST_ERR_NULL;
    if (branch && !d_branch) return ALST_ERR_NULL;
    if (!w_pre && !d_branch) return ALST_ERR_NULL;      // nothing to compute
    if ((w_pre || w_post) && !workspace) return ALST_ERR_NULL;
    if (flags & ~(ALST_FLAG_RESIDUAL_FP32 | ALST_FLAG_DW_FP32 | ALST_FLAG_DW_ACCUMULATE)) return ALST_ERR_UNSUPPORTED;
    NormParams p = {};
    p.residual = residual_out; p.branch = (const uint16_t*)branch; p.w_post = (const uint16_t*)w_post; p.gate = (const uint16_t*)gate;
    p.w_pre = (const uint16_t*)w_pre; p.d_normed = (const uint16_t*)d_normed; p.d_residual_out = d_residual_out;
    p.d_residual = d_residual; p.d_branch = (uint16_t*)d_branch; p.d_gate = (uint16_t*)d_gate; p.parts = (float*)workspace;
    p.N = N; p.scale = branch_scale; p.eps = eps; p.offset = weight_offset;
    int rc = validate_norm(p, H, gate_cols);
    if (rc == ALST_OK && !(aligned_to(dw_pre, 16) && aligned_to(dw_post, 16))) rc = ALST_ERR_ALIGN;
    if (rc == ALST_OK && (w_pre || w_post) && workspace_bytes < alst_block_norm_workspace_bytes(N, H)) rc = ALST_ERR_WORKSPACE;
    if (rc != ALST_OK) return rc;
    p.H = (int)H; p.gate_cols = (int)gate_cols;
    const NormShape s = norm_shape(H);
    const bool f32 = flags & ALST_FLAG_RESIDUAL_FP32;
    auto kernel = s.vpt == 1 ? (f32 ? norm_backward_kernel<true, 1> : norm_backward_kernel<false, 1>)
                             : (f32 ? norm_backward_kernel<true, 2> : norm_backward_kernel<false, 2>);
    const int grid = (int)norm_parts(N, H);
    const size_t lds = std::max<size_t>(2 * s.R * s.W * 2, s.R > 1 ? s.R * H : 0) * sizeof(float);
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(s.W * 64, s.R), lds, (hipStream_t)stream, p);
    if (w_pre || w_post)
        hipLaunchKernelGGL(norm_weights_kernel, dim3((unsigned)((H + 63) / 64), 2), dim3(1024), 0, (hipStream_t)stream, (const float*)p.parts,
                           grid, (int)H, dw_pre, dw_post, (flags & ALST_FLAG_DW_FP32) != 0, (flags & ALST_FLAG_DW_ACCUMULATE) != 0);
    return hipGetLastError() == hipSuccess ? ALST_OK : ALST_ERR_HIP;
}

}  // extern "C"
