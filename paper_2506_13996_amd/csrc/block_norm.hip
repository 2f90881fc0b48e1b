// The norms around a block with its gate and scaled residual addition (alst_block_norm.h), forward and backward.
//
// A row is held in the registers of W wavefronts, 8 * VPT values a lane, so that everything is read and written once; its
// sums (mean squares, and in backward the two products of a norm's gradient) go over the wavefronts through LDS.  Both are
// bound by HBM: forward at 32768 x 4096 (norms before and after, 1.07 GB) 180 us = 6.0 TB/s, backward at 256000 x 4096 (12.6 GB)
// 2.36 to 2.38 ms = 5.3 TB/s, of the 5.5 to 5.7 that a kernel reaches here that only reads four matrices and writes two.
// Values stay packed bf16 in the registers between the passes over a row (stay_packed, made_here): with the conversions and
// sums where the compiler puts them backward needs twice the registers and took 5.3 ms.
#include <algorithm>

#include "../../include/alst_block_norm.h"
#include "rowwise.h"

namespace alst {

constexpr int64_t kMaxNormH = 16384;
// Workgroups of a backward launch, each with its rows of partial weight gradients: one a compute unit.  More of them keep more
// rows open at once than memory likes: 256000 x 4096 2.34 ms, 2.54 with 512 and 2.82 with 1024 workgroups of four wavefronts.
constexpr int kMaxNormParts = 256;
constexpr int kPlaces = 2 * 16;                // of a row's sums: two turns of up to 16 wavefronts

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
    float4* lds;                               // [2][R][16]
    int turn;
    __device__ __forceinline__ RowPlace(float* lds_)
        : W(blockDim.x >> 6), R(blockDim.y), row(__builtin_amdgcn_readfirstlane(threadIdx.y)), tid(threadIdx.x),
          lds(reinterpret_cast<float4*>(lds_)), turn(0) {}
    // Sums of K values over the row: over a wavefront's lanes, then over the row's wavefronts.  The room alternates, so a
    // sum's readers are done when its room comes up again.
    template <int K>
    __device__ __forceinline__ void sum(float (&v)[K]) {
        static_assert(K <= 4, "a place holds four values");
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = wave_sum(v[k]);
        if (W == 1) return;
        float4* const at = lds + (turn * R + row) * 16;
        turn ^= 1;
        const int lane = tid & 63;
        if (lane == 0) at[tid >> 6] = make_float4(v[0], K > 1 ? v[1] : 0.f, K > 2 ? v[2] : 0.f, K > 3 ? v[3] : 0.f);
        __syncthreads();
        const float4 q = (lane & 15) < W ? at[lane & 15] : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = sum_of_16((&q.x)[k]);
    }
};

// sigmoid(z) and 1 - sigmoid(z), both to a few steps of fp32, or to 2^-126 where one of them is below that (|z| > 87; v_exp_f32 need
// not hold smaller results): from t = exp(-|z|), whose exponent is formed in two parts (v_exp_f32 is exact to a step, the product with
// log2 e is not), and 1 / (1 + t) by one step of Newton's iteration, which gives the bits of the quotient or their neighbours at a
// third of its instructions.  32768 x 5120 backward with a gate for each element, otherwise as it was then: 1302 us with expf and the
// quotient, 1173 like this.
struct Gate { float on, off; };
__device__ __forceinline__ Gate gate_of(float z) {
    constexpr float kLog2e = 1.44269502e+00f, kLog2eRest = 1.92596299e-08f, kLn2 = 6.93147182e-01f;
    float a = -fabsf(z);
    a = a < -150.f ? -150.f : a;              // (exp is 0 in fp32 from there on, and NaN stays)
    const float hi = a * kLog2e, lo = fmaf(a, kLog2eRest, fmaf(a, kLog2e, -hi));
    const float e = __builtin_amdgcn_exp2f(hi), t = fmaf(e, lo * kLn2, e);
    const float d = 1.f + t;
    float s = __builtin_amdgcn_rcpf(d);
    s = fmaf(fmaf(-d, s, 1.f), s, s);
    return z < 0.f ? Gate{t * s, s} : Gate{s, t * s};
}
__device__ __forceinline__ float bf16_value(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }

// Columns of a lane, and a weight's values there (without the weight: ones, whatever the offset).
template <int VPT>
struct Columns {
    uint32_t at[VPT];
    __device__ __forceinline__ Columns(const RowPlace& place) {
#pragma unroll
        for (int v = 0; v < VPT; ++v) at[v] = (v * (place.W * 64) + place.tid) * 8;
    }
    __device__ __forceinline__ void weight(Raw8<false> (&w)[VPT], const uint16_t* p, int H) const {
        const RowBuffer<false> row(p, 0, H, true);
#pragma unroll
        for (int v = 0; v < VPT; ++v) w[v] = p ? row.load(at[v]) : Raw8<false>{make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u)};
    }
};

// DENSE: a gate for each element.  Absent matrices read as zeros, absent weights as ones: the arithmetic has no branches.
template <bool F32, bool DENSE, int VPT, bool STREAMS>
__global__ __launch_bounds__(512) void norm_forward_kernel(NormParams p) {
    extern __shared__ float lds[];
    RowPlace at(lds);
    const Columns<VPT> col(at);
    const float inv_h = 1.f / p.H;
    const bool pre = p.w_pre != nullptr, post = p.w_post != nullptr, row_gated = !DENSE && p.gate_cols == 1;
    const float o1 = post ? p.offset : 0.f;
    Raw8<false> w1[VPT], w2[VPT];
    col.weight(w1, p.w_post, p.H);
    col.weight(w2, p.w_pre, p.H);
    for (int64_t i0 = (int64_t)blockIdx.x * at.R; i0 < p.N; i0 += (int64_t)gridDim.x * at.R) {
        const int64_t i = i0 + at.row;
        const bool row_in = i < p.N;
        const RowBuffer<F32> residual(p.residual, i, p.H, row_in), residual_out(p.residual_out, i, p.H, row_in);
        const RowBuffer<false> branch(p.branch, i, p.H, row_in), gate(DENSE ? p.gate : nullptr, i, p.H, row_in),
            normed(p.normed, i, p.H, row_in);
        Raw8<F32> r[VPT];
        Raw8<false> b[VPT], z[VPT];
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            r[v] = residual.load(col.at[v]);
            b[v] = branch.load(col.at[v]);
            if (DENSE) z[v] = gate.load(col.at[v]);
            stay_packed(w1[v]);
            stay_packed(w2[v]);
        }
        float s = p.scale;
        if (row_gated && row_in) s *= gate_of(bf16_value(p.gate + i)).on;
        if (post) {
            float bb[1] = {};
#pragma unroll
            for (int v = 0; v < VPT; ++v)
#pragma unroll
                for (int k = 0; k < 8; ++k) bb[0] = fmaf(b[v].get(k), b[v].get(k), bb[0]);
            at.sum(bb);
            s *= 1.f / sqrtf(bb[0] * inv_h + p.eps);
        }
        float x[VPT][8], xx[1] = {};
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            stay_packed(b[v]);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                float change = s * b[v].get(k) * (w1[v].get(k) + o1);
                if (DENSE) change *= gate_of(z[v].get(k)).on;
                x[v][k] = r[v].get(k) + change;
                xx[0] = fmaf(x[v][k], x[v][k], xx[0]);
            }
            residual_out.template store<STREAMS>(col.at[v], x[v]);
        }
        if (pre) {
            at.sum(xx);
            const float q2 = 1.f / sqrtf(xx[0] * inv_h + p.eps);
#pragma unroll
            for (int v = 0; v < VPT; ++v) {
                float n[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) n[k] = x[v][k] * q2 * (w2[v].get(k) + p.offset);
                normed.template store<STREAMS>(col.at[v], n);
            }
        }
    }
}

template <bool F32, bool DENSE, int VPT, bool STREAMS>
__global__ __launch_bounds__(1024) void norm_backward_kernel(NormParams p) {
    extern __shared__ float lds[];
    RowPlace at(lds);
    const Columns<VPT> col(at);
    const float inv_h = 1.f / p.H;
    const bool pre = p.w_pre != nullptr, post = p.w_post != nullptr, row_gated = !DENSE && p.gate_cols == 1;
    const float o1 = post ? p.offset : 0.f;
    Raw8<false> w1[VPT], w2[VPT];
    col.weight(w1, p.w_post, p.H);
    col.weight(w2, p.w_pre, p.H);
    float dw1[VPT][8] = {}, dw2[VPT][8] = {};
    // The next row is asked for before this one is worked on, into other registers: one workgroup a compute unit keeps the
    // memory busy, and few rows are open at a time.  (Two groups a lane leave no registers for that.)
    constexpr bool AHEAD = VPT == 1;
    struct Row {
        Raw8<F32> r[VPT], up[VPT];
        Raw8<false> dn[VPT], b[VPT], z[VPT];
        uint16_t gate;
    };
    auto load = [&](Row& row, int64_t i) {
        const bool row_in = i < p.N;
        const RowBuffer<F32> r(p.residual, i, p.H, row_in), up(p.d_residual_out, i, p.H, row_in);
        const RowBuffer<false> dn(p.d_normed, i, p.H, row_in), b(p.branch, i, p.H, row_in), z(DENSE ? p.gate : nullptr, i, p.H, row_in);
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            row.r[v] = r.load(col.at[v]);
            row.dn[v] = dn.load(col.at[v]);
            row.b[v] = b.load(col.at[v]);
            row.up[v] = up.load(col.at[v]);
            if (DENSE) row.z[v] = z.load(col.at[v]);
        }
        row.gate = row_gated && row_in ? p.gate[i] : 0;
    };
    auto work = [&](Row& row, int64_t i) {
        const bool row_in = i < p.N;
        auto &r = row.r, &up = row.up;
        auto &dn = row.dn, &b = row.b, &z = row.z;
        const RowBuffer<F32> d_residual(p.d_residual, i, p.H, row_in);
        const RowBuffer<false> d_branch(p.d_branch, i, p.H, row_in), d_gate(DENSE ? p.d_gate : nullptr, i, p.H, row_in);
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            stay_packed(w1[v]);
            stay_packed(w2[v]);
        }
        // the sums that need no other: of r'^2, of dn (w_pre + o) r', of b^2
        float s1[3] = {};
        if (pre || post) {
#pragma unroll
            for (int v = 0; v < VPT; ++v)
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float x = r[v].get(k), y = b[v].get(k);
                    s1[0] = fmaf(x, x, s1[0]);
                    s1[1] = fmaf(dn[v].get(k) * (w2[v].get(k) + p.offset), x, s1[1]);
                    s1[2] = fmaf(y, y, s1[2]);
                }
            at.sum(s1);
        }
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            stay_packed(r[v]);
            stay_packed(dn[v]);
            stay_packed(b[v]);
            stay_packed(w2[v]);
        }
        const float q2 = 1.f / sqrtf(s1[0] * inv_h + p.eps), c2 = q2 * q2 * s1[1] * inv_h;
        const float q1 = post ? 1.f / sqrtf(s1[2] * inv_h + p.eps) : 1.f;
        float g[VPT][8];                       // dr
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float x = r[v].get(k), d = dn[v].get(k);
                g[v][k] = fmaf(q2, fmaf(d, w2[v].get(k) + p.offset, -x * c2), up[v].get(k));
                dw2[v][k] = fmaf(d, x * q2, dw2[v][k]);
            }
            made_here(dw2[v]);
            d_residual.template store<STREAMS>(col.at[v], g[v]);
        }
        // dp, in g's place, and the sum over the row of dp (w_post + o) b: the norm's gradient and a row's gate both take it
        const Gate row_gate = row_gated ? gate_of(__uint_as_float((uint32_t)row.gate << 16)) : Gate{1.f, 0.f};
        const float s = p.scale * row_gate.on;
        float vb[1] = {};
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float y = b[v].get(k);
                g[v][k] *= DENSE ? s * gate_of(z[v].get(k)).on : s;
                dw1[v][k] = fmaf(g[v][k], y * q1, dw1[v][k]);
                vb[0] = fmaf(g[v][k] * (w1[v].get(k) + o1), y, vb[0]);
            }
            made_here(dw1[v]);
        }
        if (post || row_gated) at.sum(vb);
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            stay_packed(b[v]);
            stay_packed(w1[v]);
            if (DENSE && VPT > 1) stay_packed(z[v]);
        }
        if (row_gated && row_in && at.tid == 0) {
            const __bf16 dz = (__bf16)(row_gate.off * q1 * vb[0]);
            p.d_gate[i] = __builtin_bit_cast(uint16_t, dz);
        }
        const float c1 = q1 * q1 * vb[0] * inv_h;
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            float o[8], dz[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float w = w1[v].get(k) + o1, y = b[v].get(k);
                if (DENSE) dz[k] = g[v][k] * gate_of(z[v].get(k)).off * (q1 * w * y);
                const float rest = y * c1;     // (without a norm after the block left out: an infinity in b would come in as inf * 0)
                o[k] = q1 * fmaf(g[v][k], w, post ? -rest : 0.f);
            }
            d_branch.template store<STREAMS>(col.at[v], o);
            if (DENSE) d_gate.template store<STREAMS>(col.at[v], dz);
        }
    };
    const int64_t step = (int64_t)gridDim.x * at.R, first = (int64_t)blockIdx.x * at.R;
    if constexpr (AHEAD) {
        Row even, odd;
        load(even, first + at.row);
        for (int64_t i0 = first; i0 < p.N; i0 += 2 * step) {
            const int64_t i = i0 + at.row;
            load(odd, i + step);
            work(even, i);
            if (i0 + step >= p.N) break;
            load(even, i + 2 * step);
            work(odd, i + step);
        }
    } else {
        for (int64_t i0 = first; i0 < p.N; i0 += step) {
            Row row;
            load(row, i0 + at.row);
            work(row, i0 + at.row);
        }
    }
    // the rows of the workgroup together, then its partial sums of the weights' gradients
    float* const part = p.parts + (int64_t)blockIdx.x * 2 * p.H;
    for (int which = 0; which < 2; ++which) {
        if (!(which ? post : pre)) continue;
        if (at.R > 1) {
            __syncthreads();
#pragma unroll
            for (int v = 0; v < VPT; ++v)
                if (col.at[v] < (uint32_t)p.H) store8(lds + at.row * p.H, col.at[v], which ? dw1[v] : dw2[v]);
            __syncthreads();
            for (int c = at.row * blockDim.x + at.tid; c < p.H; c += blockDim.x * at.R) {
                float t = 0.f;
                for (int y = 0; y < at.R; ++y) t += lds[y * p.H + c];
                part[(int64_t)which * p.H + c] = t;
            }
        } else {
#pragma unroll
            for (int v = 0; v < VPT; ++v)
                if (col.at[v] < (uint32_t)p.H) store8(part + which * p.H, col.at[v], which ? dw1[v] : dw2[v]);
        }
    }
}

// Weight gradients: the workgroups' partial sums of 64 columns.  16 lanes take the columns of a row, so that the workgroup
// reads 64 rows at a time and a thread has its rows in flight together.
__global__ __launch_bounds__(1024) void norm_weights_kernel(const float* __restrict__ parts, int n, int H, void* dw_pre, void* dw_post,
                                                            bool f32, bool accumulate) {
    __shared__ float lds[64][64 + 4];
    const int which = blockIdx.y, x = (threadIdx.x & 15) * 4, y = threadIdx.x >> 4, c0 = blockIdx.x * 64;
    void* const out = which ? dw_post : dw_pre;
    if (!out) return;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c0 + x < H) {
#pragma unroll 8
        for (int k = y; k < n; k += 64) {
            const float4 q = *reinterpret_cast<const float4*>(parts + ((int64_t)k * 2 + which) * H + c0 + x);
            s.x += q.x; s.y += q.y; s.z += q.z; s.w += q.w;
        }
    }
    *reinterpret_cast<float4*>(&lds[y][x]) = s;
    __syncthreads();
    // 16 threads a column, four rows each, added up over lanes 64 apart
    const int c = threadIdx.x & 63, part = threadIdx.x >> 6;
    float t = lds[part * 4][c] + lds[part * 4 + 1][c] + (lds[part * 4 + 2][c] + lds[part * 4 + 3][c]);
    __syncthreads();
    lds[part][c] = t;
    __syncthreads();
    if (part == 0 && c0 + c < H) {
        t = 0.f;
        for (int k = 0; k < 16; ++k) t += lds[k][c];
        if (f32) {
            float* const o = static_cast<float*>(out) + c0 + c;
            *o = accumulate ? *o + t : t;
        } else {
            uint16_t* const o = static_cast<uint16_t*>(out) + c0 + c;
            const __bf16 r = (__bf16)(accumulate ? bf16_value(o) + t : t);
            *o = __builtin_bit_cast(uint16_t, r);
        }
    }
}

// ---- host ----

// Wavefronts of a row, rows of a workgroup, groups of eight values a lane.
struct NormShape { int W, R, vpt; };
static NormShape shape_of(int64_t H, int vpt, int waves) {
    const int W = (int)((H + 512 * vpt - 1) / (512 * vpt));
    return {W, std::max(1, waves / W), vpt};
}
// Forward: two groups a lane (5120 columns in 5 wavefronts: 32768 rows 227 us, with one group in 10 wavefronts 266; 4096 columns
// 184 and 182), one for rows of one wavefront, four above 8192 columns.
static NormShape forward_shape(int64_t H) { return shape_of(H, H <= 512 ? 1 : H <= 8192 ? 2 : 4, 4); }
// A workgroup for each row, so that the open rows are neighbours (32768 x 4096: 184 us, 209 with 2048 workgroups that walk); of short
// rows a workgroup takes several, which pays for reading the weights (262144 x 256: 98 us, 136).
static int64_t forward_grid(int64_t N, int64_t H, int R) { return std::min<int64_t>((N + R - 1) / R, H <= 512 ? 8192 : 1 << 22); }
// Backward: a group a lane, so that the wavefronts of a row spread over the four SIMDs (5120 columns: 10 wavefronts; with two
// groups 5, of which one SIMD has two: 32768 x 5120 with a gate for each element 620 us against 493) and 1024 threads have
// the registers for two rows.  Above 8192 columns two groups, and a row at a time (14731 x 10176 with a row gate: 384 us, 412 with four
// groups in half the wavefronts).  Rows of one wavefront, which wait for no other, come by 16 (262144 x 256: 184 us, 215 by 8).
static NormShape backward_shape(int64_t H) {
    return H <= 512 ? shape_of(H, 1, 16) : shape_of(H, H <= 8192 ? 1 : 2, 8);
}
using NormKernel = void (*)(NormParams);
template <bool S>
static NormKernel forward_kernel(bool f32, bool dense, int vpt) {
    static const NormKernel kernels[2][2][3] = {
        {{norm_forward_kernel<false, false, 1, S>, norm_forward_kernel<false, false, 2, S>, norm_forward_kernel<false, false, 4, S>},
         {norm_forward_kernel<false, true, 1, S>, norm_forward_kernel<false, true, 2, S>, norm_forward_kernel<false, true, 4, S>}},
        {{norm_forward_kernel<true, false, 1, S>, norm_forward_kernel<true, false, 2, S>, norm_forward_kernel<true, false, 4, S>},
         {norm_forward_kernel<true, true, 1, S>, norm_forward_kernel<true, true, 2, S>, norm_forward_kernel<true, true, 4, S>}}};
    return kernels[f32][dense][vpt >> 1];
}
template <bool S>
static NormKernel backward_kernel(bool f32, bool dense, int vpt) {
    static const NormKernel kernels[2][2][2] = {
        {{norm_backward_kernel<false, false, 1, S>, norm_backward_kernel<false, false, 2, S>},
         {norm_backward_kernel<false, true, 1, S>, norm_backward_kernel<false, true, 2, S>}},
        {{norm_backward_kernel<true, false, 1, S>, norm_backward_kernel<true, false, 2, S>},
         {norm_backward_kernel<true, true, 1, S>, norm_backward_kernel<true, true, 2, S>}}};
    return kernels[f32][dense][vpt > 1];
}
static int64_t norm_parts(int64_t N, int64_t H) {
    const NormShape s = backward_shape(H);
    return std::min<int64_t>((N + s.R - 1) / s.R, kMaxNormParts);
}

static bool norm_shape_ok(int64_t N, int64_t H) { return N >= 1 && N <= (int64_t)1 << 30 && H >= 1 && H <= kMaxNormH; }

static int validate_norm(const NormParams& p, int64_t H, int64_t gate_cols) {
    if (!norm_shape_ok(p.N, H)) return ALST_ERR_SHAPE;
    if (p.gate ? gate_cols != 1 && gate_cols != H : gate_cols != 0) return ALST_ERR_SHAPE;
    if (H % 8 != 0) return ALST_ERR_ALIGN;
    const void* ptrs[] = {p.residual, p.d_residual_out, p.branch, p.w_post, p.w_pre, p.d_normed, p.residual_out, p.d_residual, p.normed,
                          p.d_branch, p.parts};
    for (const void* q : ptrs)
        if (!aligned_to(q, 16)) return ALST_ERR_ALIGN;
    const uintptr_t gate = gate_cols == 1 ? 2 : 16;      // (a gate of one logit a row is read by elements)
    if (!aligned_to(p.gate, gate) || !aligned_to(p.d_gate, gate)) return ALST_ERR_ALIGN;
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
    p.N = N; p.eps = eps;
    p.scale = branch ? branch_scale : 0.f;                   // (absent parts are zeros and ones to the kernel,
    p.offset = w_post || w_pre ? weight_offset : 0.f;        //  whose results go by no scale or offset)
    const int rc = validate_norm(p, H, gate_cols);
    if (rc != ALST_OK) return rc;
    p.H = (int)H; p.gate_cols = (int)gate_cols;
    const NormShape s = forward_shape(H);
    const bool f32 = flags & ALST_FLAG_RESIDUAL_FP32;
    const NormKernel kernel = streams_out(N * H * 2) ? forward_kernel<true>(f32, gate_cols > 1, s.vpt)
                                                     : forward_kernel<false>(f32, gate_cols > 1, s.vpt);
    const int64_t grid = forward_grid(N, H, s.R);
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(s.W * 64, s.R), kPlaces * s.R * sizeof(float4), (hipStream_t)stream, p);
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
    p.N = N; p.scale = branch_scale; p.eps = eps;
    p.offset = w_post || w_pre ? weight_offset : 0.f;
    int rc = validate_norm(p, H, gate_cols);
    if (rc == ALST_OK && !(aligned_to(dw_pre, 16) && aligned_to(dw_post, 16))) rc = ALST_ERR_ALIGN;
    if (rc == ALST_OK && (w_pre || w_post) && workspace_bytes < alst_block_norm_workspace_bytes(N, H)) rc = ALST_ERR_WORKSPACE;
    if (rc != ALST_OK) return rc;
    p.H = (int)H; p.gate_cols = (int)gate_cols;
    // what no result contains is not read, whatever the caller passes: NaN there would reach the gradients as 0 * NaN, and the
    // branch of a block with neither norm nor gate behind it is 2 of 12 bytes an element (32768 x 4096 228 us, 299 with it)
    if (!w_pre) p.residual = nullptr;
    if (!w_post && !gate) p.branch = nullptr;
    const NormShape s = backward_shape(H);
    const bool f32 = flags & ALST_FLAG_RESIDUAL_FP32;
    const NormKernel kernel = streams_out(N * H * 2) ? backward_kernel<true>(f32, gate_cols > 1, s.vpt)
                                                     : backward_kernel<false>(f32, gate_cols > 1, s.vpt);
    const int grid = (int)norm_parts(N, H);
    const size_t lds = std::max<size_t>(kPlaces * s.R * sizeof(float4), s.R > 1 ? s.R * H * sizeof(float) : 0);
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(s.W * 64, s.R), lds, (hipStream_t)stream, p);
    if (w_pre || w_post)
        hipLaunchKernelGGL(norm_weights_kernel, dim3((unsigned)((H + 63) / 64), 2), dim3(1024), 0, (hipStream_t)stream, (const float*)p.parts,
                           grid, (int)H, dw_pre, dw_post, (flags & ALST_FLAG_DW_FP32) != 0, (flags & ALST_FLAG_DW_ACCUMULATE) != 0);
    return hipGetLastError() == hipSuccess ? ALST_OK : ALST_ERR_HIP;
}

}  // extern "C"
