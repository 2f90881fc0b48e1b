// Token embedding (alst_embedding.h): rows of a table by token, and the table's gradient by sorted tokens.
//
// The gradient: the row numbers are sorted by token (a stable radix sort, so that the rows of a token keep their order
// and the sums their bits), then runs of equal tokens are added up.  A wavefront takes kRun consecutive sorted rows and 512
// columns, keeps the sum of the run in registers and writes it out when the token changes.  A run that ends or begins
// in another wavefront's rows leaves fp32 partial sums, which join_kernel adds up.
#include <algorithm>

#include "../../include/alst_embedding.h"
#include "rowwise.h"

namespace alst {

// ---------------------------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------------------------
template <bool F32>
__global__ __launch_bounds__(256) void embedding_forward_kernel(const int32_t* __restrict__ tokens, const uint16_t* __restrict__ E,
                                                                void* __restrict__ y, int64_t N, int H, int V, int ignore_index,
                                                                float scale, int32_t* __restrict__ status) {
    // a wavefront: 512 columns of rows in turn
    const int col = blockIdx.y * 512 + (threadIdx.x & 63) * 8;
    for (int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); i < N; i += (int64_t)gridDim.x * 4) {
        const int t = tokens[i];
        const bool named = t >= 0 && t < V, kept = named && t != ignore_index;
        if (!named && t != ignore_index && status && (threadIdx.x & 63) == 0 && blockIdx.y == 0) *status = ALST_ERR_LABEL_RANGE;
        if (col >= H) continue;
        const Raw8<false> r = kept ? load8<false>(row_of<false>(E, (int64_t)t * H), col) : zero8<false>();
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = kept ? r.get(k) * scale : 0.f;
        store8<F32>(row_of<F32>(y, i * H), col, v);
    }
}

// ---------------------------------------------------------------------------------------------
// the sort
// ---------------------------------------------------------------------------------------------
constexpr int kDigitBits = 9;                  // two passes for a vocabulary below 2^18 = 262144, three beyond
constexpr int kDigits = 1 << kDigitBits;
constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kMostSortBlocks = 256;

struct Pair { int32_t key, row; };             // key: the token, V for one that takes no part

struct EmbeddingHeader { int32_t status; int32_t pad[63]; };

__global__ void embedding_header_kernel(EmbeddingHeader* h) {
    if (threadIdx.x < 64) h->pad[threadIdx.x ? threadIdx.x - 1 : 0] = 0;
    if (threadIdx.x == 0) h->status = 0;
}

// Where a pass of the sort finds its keys: the first in the tokens, later ones in the pairs of the pass before.
struct SortSource {
    const int32_t* tokens;
    const Pair* pairs;
    int V, ignore_index;
    __device__ __forceinline__ Pair get(int64_t i, int32_t* status) const {
        if (pairs) return pairs[i];
        const int t = tokens[i];
        const bool named = t >= 0 && t < V;
        if (!named && t != ignore_index && status) *status = ALST_ERR_LABEL_RANGE;
        return {named && t != ignore_index ? t : V, (int32_t)i};
    }
};

// counts[block][digit]: the keys of a workgroup's share of the rows.
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(SortSource src, int64_t N, int64_t share, int shift,
                                                                  uint32_t* __restrict__ counts, int32_t* __restrict__ status) {
    __shared__ uint32_t lds[kDigits];
    for (int d = threadIdx.x; d < kDigits; d += kSortThreads) lds[d] = 0;
    __syncthreads();
    const int64_t from = (int64_t)blockIdx.x * share, upto = min(from + share, N);
    for (int64_t i = from + threadIdx.x; i < upto; i += kSortThreads)
        atomicAdd(&lds[(src.get(i, status).key >> shift) & (kDigits - 1)], 1u);
    __syncthreads();
    for (int d = threadIdx.x; d < kDigits; d += kSortThreads) counts[(int64_t)blockIdx.x * kDigits + d] = lds[d];
}

// Puts the workgroup's keys behind those of smaller digits and those of the same digit before them.
__global__ __launch_bounds__(kSortThreads) void sort_scatter_kernel(SortSource src, Pair* __restrict__ to, int64_t N, int64_t share,
                                                                    int shift, const uint32_t* __restrict__ counts) {
    __shared__ uint32_t place[kSortWaves][kDigits];      // next place of a wavefront's next key of a digit
    __shared__ uint32_t sums[kSortWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int d = threadIdx.x; d < kSortWaves * kDigits; d += kSortThreads) (&place[0][0])[d] = 0;
    __syncthreads();
    // a wavefront's keys are consecutive
    const int64_t block0 = (int64_t)blockIdx.x * share, each = share / kSortWaves;
    const int64_t from = min(block0 + wave * each, N), upto = min(from + each, N);
    for (int64_t i = from + lane; i < upto; i += 64) atomicAdd(&place[wave][(src.get(i, nullptr).key >> shift) & (kDigits - 1)], 1u);
    __syncthreads();
    // first place of this workgroup's keys of digit threadIdx.x
    uint32_t before = 0, all = 0;
    if (threadIdx.x < kDigits) {
        for (uint32_t b = 0; b < gridDim.x; ++b) {
            const uint32_t n = counts[(int64_t)b * kDigits + threadIdx.x];
            if (b < blockIdx.x) before += n;
            all += n;
        }
    }
    uint32_t incl = all;                                 // sum over the digits up to this one
    for (int step = 1; step < 64; step <<= 1) {
        const uint32_t o = __shfl_up(incl, step);
        if (lane >= step) incl += o;
    }
    if (lane == 63) sums[wave] = incl;
    __syncthreads();
    for (int w = 0; w < wave; ++w) incl += sums[w];
    if (threadIdx.x < kDigits) {
        uint32_t at = incl - all + before;
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t n = place[w][threadIdx.x];
            place[w][threadIdx.x] = at;
            at += n;
        }
    }
    __syncthreads();
    volatile uint32_t* const mine = place[wave];
    for (int64_t i0 = from; i0 < upto; i0 += 64) {
        const bool have = i0 + lane < upto;
        const Pair p = have ? src.get(i0 + lane, nullptr) : Pair{0, 0};
        const int d = (p.key >> shift) & (kDigits - 1);
        uint64_t same = __ballot(have);                  // the lanes with this digit
#pragma unroll
        for (int b = 0; b < kDigitBits; ++b) {
            const uint64_t set = __ballot(d >> b & 1);
            same &= d >> b & 1 ? set : ~set;
        }
        const int rank = __popcll(same & (((uint64_t)1 << lane) - 1));
        uint32_t at = 0;
        if (have) at = mine[d] + rank;
        __builtin_amdgcn_wave_barrier();
        if (have && rank == 0) mine[d] = at + __popcll(same);
        __builtin_amdgcn_wave_barrier();
        if (have) to[at] = p;
    }
}

// ---------------------------------------------------------------------------------------------
// the sums
// ---------------------------------------------------------------------------------------------
constexpr int kRun = 32;                       // sorted rows of a wavefront

struct Grad {
    void* dE;
    float scale;
    bool f32, accumulate;
};

__device__ __forceinline__ void write_grad(const Grad& g, int64_t at, const float (&sum)[8]) {
    float v[8];
    if (g.f32) {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = sum[k] * g.scale;
        if (g.accumulate) {
            const Raw8<true> old = load8<true>(row_of<true>(g.dE, at), 0);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] += old.get(k);
        }
        store8<true>(row_of<true>(g.dE, at), 0, v);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = sum[k] * g.scale;
        if (g.accumulate) {
            const Raw8<false> old = load8<false>(row_of<false>(g.dE, at), 0);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] += old.get(k);
        }
        store8<false>(row_of<false>(g.dE, at), 0, v);
    }
}

__global__ __launch_bounds__(256) void zero_rows_kernel(uint4* __restrict__ p, int64_t lines) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < lines; i += (int64_t)gridDim.x * 256) p[i] = make_uint4(0, 0, 0, 0);
}

// parts[range][0]: sum of the range's rows of the token that came over from the range before; [1]: of the token that goes on
// in the next range and began in this one.
template <bool F32>
__global__ __launch_bounds__(256) void run_sums_kernel(const Pair* __restrict__ pairs, const void* __restrict__ dy, int64_t N, int H,
                                                       int V, float* __restrict__ parts, Grad g) {
    const int lane = threadIdx.x & 63, col = blockIdx.y * 512 + lane * 8;
    const int64_t range = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), p0 = range * kRun;
    if (p0 >= N) return;
    const int rows = (int)min((int64_t)kRun, N - p0);
    Pair mine = {V, 0};
    if (lane < rows) mine = pairs[p0 + lane];
    const int prev = p0 > 0 ? pairs[p0 - 1].key : -1, next = p0 + rows < N ? pairs[p0 + rows].key : V;
    float sum[8] = {};
    bool came = __builtin_amdgcn_readlane(mine.key, 0) == prev;
    for (int j0 = 0; j0 < rows; j0 += 8) {
        Raw8<F32> r[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int key = __builtin_amdgcn_readlane(mine.key, j0 + j), row = __builtin_amdgcn_readlane(mine.row, j0 + j);
            r[j] = key < V && col < H ? load8<F32>(row_of<F32>(dy, (int64_t)row * H), col) : zero8<F32>();
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int at = j0 + j;
            const int key = __builtin_amdgcn_readlane(mine.key, at);
            if (key >= V) return;                        // (no rows behind the last token's)
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[k] += r[j].get(k);
            const int behind = at + 1 < rows ? __builtin_amdgcn_readlane(mine.key, (at + 1) & 63) : next;
            const bool last = at + 1 == rows;
            if (key == behind && !last) continue;
            if (col < H) {
                if (came) store8<true>(parts + range * 2 * H, col, sum);
                else if (key == behind) store8<true>(parts + (range * 2 + 1) * H, col, sum);
                else write_grad(g, (int64_t)key * H + col, sum);
            }
            if (last) return;
            came = false;
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[k] = 0.f;
        }
    }
}

// A token whose rows lie in several ranges: the partial sums of the range where it begins and of those behind it.
__global__ __launch_bounds__(64) void join_kernel(const Pair* __restrict__ pairs, int64_t N, int H, int V, const float* __restrict__ parts,
                                                  Grad g) {
    const int lane = threadIdx.x, col = blockIdx.y * 512 + lane * 8;
    const int64_t range = blockIdx.x, p0 = range * kRun, end = p0 + kRun;
    if (end >= N) return;
    const int key = pairs[end - 1].key;
    if (key >= V || pairs[end].key != key) return;                              // does not go on
    if (p0 > 0 && pairs[p0].key == key && pairs[p0 - 1].key == key) return;      // did not begin here
    float sum[8] = {};
    auto add = [&](int64_t slot) {
        if (col >= H) return;
        const Raw8<true> r = load8<true>(parts + slot * H, col);
#pragma unroll
        for (int k = 0; k < 8; ++k) sum[k] += r.get(k);
    };
    // (a run that fills its first range from the first row on is that range's slot 1 too)
    add(range * 2 + 1);
    for (int64_t r = range + 1; r * kRun < N && pairs[r * kRun].key == key; ++r) add(r * 2);
    if (col < H) write_grad(g, (int64_t)key * H + col, sum);
}

// ---------------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------------
struct EmbeddingLayout {
    int64_t share;               // rows of a workgroup of the sort, whole wavefronts' worth
    int blocks, passes;
    size_t counts, pairs[2], parts, total;
};

static EmbeddingLayout make_embedding_layout(int64_t N, int64_t H, int64_t V) {
    EmbeddingLayout L = {};
    auto up = [](int64_t v, int64_t to) { return (v + to - 1) / to * to; };
    L.share = up(std::max((N + kMostSortBlocks - 1) / kMostSortBlocks, (int64_t)4 * kSortThreads), kSortThreads);
    L.blocks = (int)((N + L.share - 1) / L.share);
    int bits = 1;
    while (V >> bits) ++bits;                            // of the largest key, V
    L.passes = (bits + kDigitBits - 1) / kDigitBits;
    size_t o = sizeof(EmbeddingHeader);
    auto take = [&](size_t bytes) { size_t at = o; o = (size_t)up((int64_t)(o + bytes), 256); return at; };
    L.counts = take((size_t)kMostSortBlocks * kDigits * 4);
    L.pairs[0] = take((size_t)N * sizeof(Pair));
    L.pairs[1] = take((size_t)N * sizeof(Pair));
    L.parts = take((size_t)((N + kRun - 1) / kRun) * 2 * H * 4);
    L.total = o;
    return L;
}

static bool embedding_shape_ok(int64_t N, int64_t H, int64_t V) {
    return N >= 1 && N <= (int64_t)1 << 30 && H >= 1 && H <= (int64_t)1 << 20 && V >= 1 && V <= (int64_t)1 << 24;
}

}  // namespace alst

using namespace alst;

extern "C" {

size_t alst_embedding_workspace_bytes(int64_t N, int64_t H, int64_t V) {
    return embedding_shape_ok(N, H, V) ? make_embedding_layout(N, H, V).total : 0;
}

int alst_embedding_forward(const int32_t* tokens, const void* E, int64_t N, int64_t H, int64_t V, int32_t ignore_index, float scale,
                           void* y, int32_t* device_status_out, uint32_t flags, void* stream) {
    if (!tokens || !E || !y) return ALST_ERR_NULL;
    if (flags & ~ALST_FLAG_RESIDUAL_FP32) return ALST_ERR_UNSUPPORTED;
    if (!embedding_shape_ok(N, H, V)) return ALST_ERR_SHAPE;
    if (H % 8 != 0 || !aligned_to(tokens, 16) || !aligned_to(E, 16) || !aligned_to(y, 16) || !aligned_to(device_status_out, 4))
        return ALST_ERR_ALIGN;
    const dim3 grid((unsigned)std::min<int64_t>((N + 3) / 4, 1 << 20), (unsigned)((H + 511) / 512));
    auto kernel = flags & ALST_FLAG_RESIDUAL_FP32 ? embedding_forward_kernel<true> : embedding_forward_kernel<false>;
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, (hipStream_t)stream, tokens, (const uint16_t*)E, y, N, (int)H, (int)V,
                       ignore_index, scale, device_status_out);
    return hipGetLastError() == hipSuccess ? ALST_OK : ALST_ERR_HIP;
}

int alst_embedding_backward(const int32_t* tokens, const void* dy, int64_t N, int64_t H, int64_t V, int32_t ignore_index, float scale,
                            void* dE, void* workspace, size_t workspace_bytes, uint32_t flags, void* stream) {
    if (!tokens || !dy || !dE || !workspace) return ALST_ERR_NULL;
    if (flags & ~(ALST_FLAG_RESIDUAL_FP32 | ALST_FLAG_DW_FP32 | ALST_FLAG_DW_ACCUMULATE)) return ALST_ERR_UNSUPPORTED;
    if (!embedding_shape_ok(N, H, V)) return ALST_ERR_SHAPE;
    if (H % 8 != 0 || !aligned_to(tokens, 16) || !aligned_to(dy, 16) || !aligned_to(dE, 16) || !aligned_to(workspace, 16))
        return ALST_ERR_ALIGN;
    const EmbeddingLayout L = make_embedding_layout(N, H, V);
    if (workspace_bytes < L.total) return ALST_ERR_WORKSPACE;
    const hipStream_t s = (hipStream_t)stream;
    unsigned char* const ws = static_cast<unsigned char*>(workspace);
    EmbeddingHeader* const header = reinterpret_cast<EmbeddingHeader*>(ws);
    uint32_t* const counts = reinterpret_cast<uint32_t*>(ws + L.counts);
    float* const parts = reinterpret_cast<float*>(ws + L.parts);
    const Grad g = {dE, scale, (flags & ALST_FLAG_DW_FP32) != 0, (flags & ALST_FLAG_DW_ACCUMULATE) != 0};

    hipLaunchKernelGGL(embedding_header_kernel, dim3(1), dim3(64), 0, s, header);
    if (!g.accumulate) {
        const int64_t lines = V * H * (g.f32 ? 4 : 2) / 16;
        hipLaunchKernelGGL(zero_rows_kernel, dim3((unsigned)std::min<int64_t>((lines + 255) / 256, 4096)), dim3(256), 0, s,
                           static_cast<uint4*>(dE), lines);
    }
    SortSource src = {tokens, nullptr, (int)V, ignore_index};
    for (int pass = 0; pass < L.passes; ++pass) {
        Pair* const to = reinterpret_cast<Pair*>(ws + L.pairs[pass & 1]);
        hipLaunchKernelGGL(sort_count_kernel, dim3(L.blocks), dim3(kSortThreads), 0, s, src, N, L.share, pass * kDigitBits, counts,
                           &header->status);
        hipLaunchKernelGGL(sort_scatter_kernel, dim3(L.blocks), dim3(kSortThreads), 0, s, src, to, N, L.share, pass * kDigitBits,
                           (const uint32_t*)counts);
        src.pairs = to;
    }
    const unsigned slabs = (unsigned)((H + 511) / 512);
    const int64_t ranges = (N + kRun - 1) / kRun;
    auto sums = flags & ALST_FLAG_RESIDUAL_FP32 ? run_sums_kernel<true> : run_sums_kernel<false>;
    hipLaunchKernelGGL(sums, dim3((unsigned)((ranges + 3) / 4), slabs), dim3(256), 0, s, src.pairs, dy, N, (int)H, (int)V, parts, g);
    hipLaunchKernelGGL(join_kernel, dim3((unsigned)ranges, slabs), dim3(64), 0, s, src.pairs, N, (int)H, (int)V, (const float*)parts, g);
    return hipGetLastError() == hipSuccess ? ALST_OK : ALST_ERR_HIP;
}

}  // extern "C"
