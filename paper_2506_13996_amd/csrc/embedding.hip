// Token embedding (alst_embedding.h): rows of a table by token, and the table's gradient by sorted tokens.
//
// The gradient: the row numbers are sorted by token (a stable radix sort, so that the rows of a token keep their order
// and the sums their bits), then runs of equal tokens are added up.  A wavefront takes `run` consecutive sorted rows and 512
// columns (the wavefronts of a workgroup the columns of the same rows), keeps the sum of a token's rows in registers and
// writes it out when the token changes.  A token whose rows go on in another range leaves fp32 partial sums, which
// join_kernel adds up.  Rows of tokens that do not occur are filled with zeros beside the sort and the sums.
#include <algorithm>

#include "../../include/alst_embedding.h"
#include "rowwise.h"

namespace alst {

// ---------------------------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------------------------
constexpr int64_t kMostGroups = 1 << 22;        // workgroups of a launch (their threads have to stay below 2^32); more work is walked

constexpr int kForwardColumns = 1024;          // of a wavefront: two groups of eight values a lane
constexpr int kForwardRows = 4;                // rows of a wavefront, in flight together

// W wavefronts (blockDim.x / 64) take kForwardRows rows, 1024 columns each; the R rows of wavefronts of a workgroup lie behind
// each other.  A token that takes no part has no row: it is read as zeros.
template <bool F32>
__global__ __launch_bounds__(256) void embedding_forward_kernel(const int32_t* __restrict__ tokens, const uint16_t* __restrict__ E,
                                                                void* __restrict__ y, int64_t N, int H, int V, int ignore_index,
                                                                float scale, int32_t* __restrict__ status) {
    const uint32_t next = blockDim.x * 8, col = blockIdx.y * 2 * next + threadIdx.x * 8;
    const int64_t rows = (int64_t)blockDim.y * kForwardRows;
    for (int64_t g0 = blockIdx.x * rows; g0 < N; g0 += gridDim.x * rows) {
        const int64_t i0 = g0 + __builtin_amdgcn_readfirstlane(threadIdx.y) * kForwardRows;
        Raw8<false> r[kForwardRows][2];
#pragma unroll
        for (int j = 0; j < kForwardRows; ++j) {
            const int64_t i = i0 + j;
            const int t = __builtin_amdgcn_readfirstlane(i < N ? tokens[i] : ignore_index);
            const bool named = t >= 0 && t < V;
            if (!named && t != ignore_index && status && threadIdx.x == 0 && blockIdx.y == 0) *status = ALST_ERR_LABEL_RANGE;
            const RowBuffer<false> row(E, t, H, named && t != ignore_index);
            r[j][0] = row.load(col);
            r[j][1] = row.load(col + next);
        }
#pragma unroll
        for (int j = 0; j < kForwardRows; ++j) {
            const RowBuffer<F32> row(y, i0 + j, H, i0 + j < N);
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float v[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = r[j][c].get(k) * scale;
                row.store(col + c * next, v);
            }
        }
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

// Zeros for the status word, the second pass's counts and (occurs) the marks of the tokens that occur.
__global__ __launch_bounds__(256) void embedding_clear_kernel(uint4* __restrict__ p, int64_t lines) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < lines; i += (int64_t)gridDim.x * 256) p[i] = make_uint4(0, 0, 0, 0);
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

// Rows from..upto-1 of dE without a token are filled with zeros, by wavefront `wave` of `waves`.
struct ZeroRows {
    void* dE;
    const uint8_t* occurs;       // [V]
    int64_t from, upto;
    int H;
    bool f32;
    template <bool F32>
    __device__ __forceinline__ void fill(int v) const {
        const RowBuffer<F32> row(dE, v, H, true);
        const float zeros[8] = {};
        for (int c = (threadIdx.x & 63) * 8; c < H; c += 512) row.store(c, zeros);
    }
    __device__ __forceinline__ void run(int64_t wave, int64_t waves) const {
        constexpr int kTogether = 16;
        for (int64_t v0 = from + wave * kTogether; v0 < upto; v0 += waves * kTogether) {
            const int lane = threadIdx.x & 63;
            const uint64_t absent = __ballot(lane < kTogether && v0 + lane < upto && !occurs[v0 + lane]);
            for (uint64_t rest = absent; rest; rest &= rest - 1) {
                const int v = (int)v0 + __builtin_ctzll(rest);
                if (f32) fill<true>(v);
                else fill<false>(v);
            }
        }
    }
};

// counts[block][digit]: the keys of a workgroup's share of the rows.  occurs (or NULL): marks the tokens.
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(SortSource src, int64_t N, int64_t share, uint32_t* __restrict__ counts,
                                                                  uint8_t* __restrict__ occurs, int32_t* __restrict__ status) {
    __shared__ uint32_t lds[kDigits];
    for (int d = threadIdx.x; d < kDigits; d += kSortThreads) lds[d] = 0;
    __syncthreads();
    const int64_t from = (int64_t)blockIdx.x * share, upto = min(from + share, N);
    for (int64_t i = from + threadIdx.x; i < upto; i += kSortThreads) {
        const int key = src.get(i, status).key;
        atomicAdd(&lds[key & (kDigits - 1)], 1u);
        if (occurs && key < src.V) occurs[key] = 1;
    }
    __syncthreads();
    for (int d = threadIdx.x; d < kDigits; d += kSortThreads) counts[(int64_t)blockIdx.x * kDigits + d] = lds[d];
}

struct SortRoom {
    uint32_t place[kSortWaves][kDigits];      // next place of a wavefront's next key of a digit
    uint32_t sums[kSortWaves];
};

// Puts the keys of a workgroup (`block` of `blocks`) behind those of smaller digits and those of the same digit before
// them.  counts: those of all workgroups (NULL: there is one).  later: the next pass's counts, added to (NULL: none).
__device__ __forceinline__ void sort_scatter(const SortSource& src, Pair* __restrict__ to, int64_t N, int share_bits, int shift,
                                             const uint32_t* __restrict__ counts, uint32_t* __restrict__ later, int block, int blocks,
                                             SortRoom& room, int32_t* status) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int d = threadIdx.x; d < kSortWaves * kDigits; d += kSortThreads) (&room.place[0][0])[d] = 0;
    __syncthreads();
    // a wavefront's keys are consecutive
    const int64_t share = (int64_t)1 << share_bits, each = share / kSortWaves;
    const int64_t from = min(block * share + wave * each, N), upto = min(from + each, N);
    for (int64_t i = from + lane; i < upto; i += 64) atomicAdd(&room.place[wave][(src.get(i, status).key >> shift) & (kDigits - 1)], 1u);
    // first place of this workgroup's keys of digit threadIdx.x
    uint32_t before = 0, all = 0;
    if (counts && threadIdx.x < kDigits) {
#pragma unroll 16
        for (int b = 0; b < blocks; ++b) {
            const uint32_t n = counts[(int64_t)b * kDigits + threadIdx.x];
            before += b < block ? n : 0;
            all += n;
        }
    }
    __syncthreads();
    if (!counts && threadIdx.x < kDigits)
        for (int w = 0; w < kSortWaves; ++w) all += room.place[w][threadIdx.x];
    uint32_t incl = all;                                 // sum over the digits up to this one
    for (int step = 1; step < 64; step <<= 1) {
        const uint32_t o = __shfl_up(incl, step);
        if (lane >= step) incl += o;
    }
    if (lane == 63) room.sums[wave] = incl;
    __syncthreads();
    for (int w = 0; w < wave; ++w) incl += room.sums[w];
    if (threadIdx.x < kDigits) {
        uint32_t at = incl - all + before;
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t n = room.place[w][threadIdx.x];
            room.place[w][threadIdx.x] = at;
            at += n;
        }
    }
    __syncthreads();
    volatile uint32_t* const mine = room.place[wave];
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
        if (have) {
            to[at] = p;
            // (whole numbers: the order of these additions changes nothing)
            if (later) atomicAdd(&later[((int64_t)(at >> share_bits)) * kDigits + ((p.key >> (shift + kDigitBits)) & (kDigits - 1))], 1u);
        }
    }
}

// A pass, and beside it (workgroups from `blocks` on) rows of zeros.
__global__ __launch_bounds__(kSortThreads) void sort_scatter_kernel(SortSource src, Pair* __restrict__ to, int64_t N, int share_bits,
                                                                    int shift, const uint32_t* __restrict__ counts,
                                                                    uint32_t* __restrict__ later, int blocks, ZeroRows zeros) {
    __shared__ SortRoom room;
    if ((int)blockIdx.x >= blocks) {
        zeros.run((int64_t)(blockIdx.x - blocks) * kSortWaves + (threadIdx.x >> 6), (int64_t)(gridDim.x - blocks) * kSortWaves);
        return;
    }
    sort_scatter(src, to, N, share_bits, shift, counts, later, blockIdx.x, blocks, room, nullptr);
}

// All of the sort where one workgroup's share holds the rows: every pass, the marks of the tokens and the status word.
__global__ __launch_bounds__(kSortThreads) void sort_short_kernel(SortSource src, Pair* a, Pair* b, int64_t N, int share_bits, int passes,
                                                                  uint8_t* occurs, int64_t occurs_lines, EmbeddingHeader* header) {
    __shared__ SortRoom room;
    if (threadIdx.x < sizeof(EmbeddingHeader) / 4) reinterpret_cast<int32_t*>(header)[threadIdx.x] = 0;
    if (occurs) {
        uint4* const lines = reinterpret_cast<uint4*>(occurs);
        for (int64_t i = threadIdx.x; i < occurs_lines; i += kSortThreads) lines[i] = make_uint4(0, 0, 0, 0);
    }
    __syncthreads();
    for (int pass = 0; pass < passes; ++pass) {
        sort_scatter(src, pass & 1 ? b : a, N, share_bits, pass * kDigitBits, nullptr, nullptr, 0, 1, room, pass ? nullptr : &header->status);
        src.pairs = pass & 1 ? b : a;
        __threadfence_block();
        __syncthreads();
    }
    if (occurs)
        for (int64_t i = threadIdx.x; i < N; i += kSortThreads) {
            const int key = src.pairs[i].key;
            if (key < src.V) occurs[key] = 1;
        }
}

// ---------------------------------------------------------------------------------------------
// the sums
// ---------------------------------------------------------------------------------------------
struct Grad {
    void* dE;
    float scale;
    bool f32, accumulate;
};

template <bool F32>
__device__ __forceinline__ void write_grad_as(const Grad& g, int key, int H, uint32_t col, const float (&sum)[8]) {
    const RowBuffer<F32> row(g.dE, key, H, true);
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = sum[k] * g.scale;
    if (g.accumulate) {
        const Raw8<F32> old = row.load(col);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] += old.get(k);
    }
    row.store(col, v);
}
__device__ __forceinline__ void write_grad(const Grad& g, int key, int H, uint32_t col, const float (&sum)[8]) {
    if (g.f32) write_grad_as<true>(g, key, H, col, sum);
    else write_grad_as<false>(g, key, H, col, sum);
}

constexpr int kSumThreads = 512;
constexpr int kRowsTogether = 8;               // rows of dy that a wavefront has in flight
constexpr int kJoinThreads = 256;

// parts[range][0]: sum of the range's rows of the token that came over from the range before; [1]: of the token that goes on
// in the next range and began in this one.  A workgroup: a range (run <= 64 rows) and 512 columns a wavefront; workgroups from
// `ranges` on: rows of zeros.
template <bool F32>
__global__ __launch_bounds__(kSumThreads) void run_sums_kernel(const Pair* __restrict__ pairs, const void* __restrict__ dy, int64_t N,
                                                               int H, int V, int run, int64_t ranges, float* __restrict__ parts, Grad g,
                                                               ZeroRows zeros) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int64_t range = blockIdx.x, p0 = range * run;
    if (range >= ranges) {
        zeros.run(((range - ranges) * gridDim.y + blockIdx.y) * waves + wave, (int64_t)(gridDim.x - ranges) * gridDim.y * waves);
        return;
    }
    const uint32_t col = (blockIdx.y * waves + wave) * 512 + lane * 8;
    const int rows = (int)min((int64_t)run, N - p0);
    Pair mine = {V, 0};
    if (lane < rows) mine = pairs[p0 + lane];
    const int prev = p0 > 0 ? pairs[p0 - 1].key : -1, next = p0 + rows < N ? pairs[p0 + rows].key : V;
    float sum[8] = {};
    bool came = __builtin_amdgcn_readlane(mine.key, 0) == prev;
    for (int j0 = 0; j0 < rows; j0 += kRowsTogether) {
        Raw8<F32> r[kRowsTogether];
#pragma unroll
        for (int j = 0; j < kRowsTogether; ++j) {
            const int key = __builtin_amdgcn_readlane(mine.key, j0 + j), row = __builtin_amdgcn_readlane(mine.row, j0 + j);
            r[j] = RowBuffer<F32>(dy, row, H, key < V).load(col);
        }
#pragma unroll
        for (int j = 0; j < kRowsTogether; ++j) {
            const int at = j0 + j;
            const int key = __builtin_amdgcn_readlane(mine.key, at);
            if (key >= V) return;                        // (no rows behind the last token's)
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[k] += r[j].get(k);
            const bool last = at + 1 == rows;
            const int behind = last ? next : __builtin_amdgcn_readlane(mine.key, (at + 1) & 63);
            if (key == behind && !last) continue;
            if (came) RowBuffer<true>(parts, range * 2, H, true).store(col, sum);
            else if (key == behind) RowBuffer<true>(parts, range * 2 + 1, H, true).store(col, sum);
            else write_grad(g, key, H, col, sum);
            if (last) return;
            came = false;
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[k] = 0.f;
        }
    }
}

// A token whose rows lie in several ranges: the partial sums of the range where it begins (slot 1, also if the range holds nothing
// else) and of those behind it (slot 0).  Many of them are dealt to the wavefronts of the workgroup in turn.
__global__ __launch_bounds__(kJoinThreads) void join_kernel(const Pair* __restrict__ pairs, int64_t N, int H, int V, int run, int64_t ranges,
                                                            const float* __restrict__ parts, Grad g) {
    constexpr int kWaves = kJoinThreads / 64;
    __shared__ float lds[kWaves][512];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t col = blockIdx.y * 512 + lane * 8;
    for (int64_t range = blockIdx.x; range + 1 < ranges; range += gridDim.x) {
        const int64_t p0 = range * run, end = p0 + run;
        const int key = __builtin_amdgcn_readfirstlane(pairs[end - 1].key);
        if (key >= V || pairs[end].key != key) continue;                              // does not go on
        if (p0 > 0 && pairs[p0].key == key && pairs[p0 - 1].key == key) continue;      // did not begin here
        int64_t more = 0;                                    // ranges behind that begin with it
        for (int n = kJoinThreads; n == kJoinThreads; more += n) {
            const int64_t r = range + 1 + more + threadIdx.x;
            n = __syncthreads_count(r < ranges && pairs[r * run].key == key);
        }
        float sum[8] = {};
        auto add = [&](int64_t first, int64_t step) {
#pragma unroll 4
            for (int64_t k = first; k <= more; k += step) {
                const Raw8<true> r = RowBuffer<true>(parts, (range + k) * 2 + (k == 0), H, true).load(col);
#pragma unroll
                for (int j = 0; j < 8; ++j) sum[j] += r.get(j);
            }
        };
        if (more < 2 * kWaves) {
            if (wave == 0) add(0, 1);
        } else {
            add(wave, kWaves);
            if (wave != 0) store8<true>(lds[wave], lane * 8, sum);
            __syncthreads();
            if (wave == 0) {
#pragma unroll
                for (int w = 1; w < kWaves; ++w) {
                    const Raw8<true> r = load8<true>(lds[w], lane * 8);
#pragma unroll
                    for (int j = 0; j < 8; ++j) sum[j] += r.get(j);
                }
            }
            __syncthreads();
        }
        if (wave == 0) write_grad(g, key, H, col, sum);
    }
}

// ---------------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------------
constexpr int64_t kZerosBesidePass = (int64_t)64 << 20;
constexpr int kShortBits = 12;                 // up to 4096 rows are sorted by one workgroup

struct EmbeddingLayout {
    int share_bits;              // rows of a workgroup of the sort: 2^share_bits
    int blocks, passes, run;
    int64_t ranges, occurs_bytes;
    // header and counts of the passes behind the first and the marks of the tokens (zeros at the start, to `cleared`), counts of the
    // first pass, pairs, partial sums
    size_t later[2], occurs, cleared, counts, pairs[2], parts, total;
};

static int slabs_of(int64_t H) { return (int)((H + 511) / 512); }

// Sorted rows of a wavefront: 64, fewer where that leaves less than 4096 wavefronts.
static int run_of(int64_t N, int64_t H) {
    int run = 64;
    while (run > 8 && N * slabs_of(H) < (int64_t)run * 4096) run /= 2;
    return run;
}

static EmbeddingLayout make_embedding_layout(int64_t N, int64_t H, int64_t V) {
    EmbeddingLayout L = {};
    auto up = [](int64_t v, int64_t to) { return (v + to - 1) / to * to; };
    L.share_bits = kShortBits;
    while ((N + ((int64_t)1 << L.share_bits) - 1) >> L.share_bits > kMostSortBlocks) ++L.share_bits;
    L.blocks = (int)((N + ((int64_t)1 << L.share_bits) - 1) >> L.share_bits);
    int bits = 1;
    while (V >> bits) ++bits;                            // of the largest key, V
    L.passes = (bits + kDigitBits - 1) / kDigitBits;
    L.run = run_of(N, H);
    L.ranges = (N + L.run - 1) / L.run;
    size_t o = sizeof(EmbeddingHeader);
    auto take = [&](size_t bytes) { size_t at = o; o = (size_t)up((int64_t)(o + bytes), 256); return at; };
    const size_t counts = (size_t)kMostSortBlocks * kDigits * 4;
    for (int k = 0; k < 2; ++k) L.later[k] = take(counts);
    L.occurs = take((size_t)V);
    L.occurs_bytes = (int64_t)(o - L.occurs);
    L.cleared = o;
    L.counts = take(counts);
    L.pairs[0] = take((size_t)N * sizeof(Pair));
    L.pairs[1] = take((size_t)N * sizeof(Pair));
    // (runs get longer with N: room for the partial sums of every shorter call)
    int64_t ranges = 0;
    for (int run = 8; run <= L.run; run *= 2) {
        const int64_t most = run < 64 ? std::min(N, ((int64_t)run * 2 * 4096 - 1) / slabs_of(H) ) : N;
        ranges = std::max(ranges, (most + run - 1) / run);
    }
    L.parts = take((size_t)ranges * 2 * H * 4);
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
    const int W = (int)std::min<int64_t>((H + kForwardColumns - 1) / kForwardColumns, 4), R = 4 / W;
    const int64_t rows = (int64_t)R * kForwardRows, columns = (int64_t)W * kForwardColumns;
    const dim3 grid((unsigned)std::min((N + rows - 1) / rows, kMostGroups), (unsigned)((H + columns - 1) / columns));
    auto kernel = flags & ALST_FLAG_RESIDUAL_FP32 ? embedding_forward_kernel<true> : embedding_forward_kernel<false>;
    hipLaunchKernelGGL(kernel, grid, dim3(W * 64, R), 0, (hipStream_t)stream, tokens, (const uint16_t*)E, y, N, (int)H, (int)V,
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
    float* const parts = reinterpret_cast<float*>(ws + L.parts);
    const Grad g = {dE, scale, (flags & ALST_FLAG_DW_FP32) != 0, (flags & ALST_FLAG_DW_ACCUMULATE) != 0};
    uint8_t* const occurs = g.accumulate ? nullptr : ws + L.occurs;
    // rows of zeros: a share beside each pass of the sort that moves rows (whose few workgroups leave the memory idle for about
    // kZerosBesidePass bytes' time), the rest beside the sums
    ZeroRows zeros = {dE, occurs, 0, 0, (int)H, g.f32};
    const int64_t row_bytes = H * (g.f32 ? 4 : 2);
    auto take_zeros = [&](int64_t bytes) {               // workgroups of 16 wavefronts that fill the next `bytes`
        zeros.from = zeros.upto;
        if (g.accumulate) return 0;
        zeros.upto = std::min<int64_t>(V, zeros.from + (bytes + row_bytes - 1) / row_bytes);
        return (int)std::min<int64_t>((zeros.upto - zeros.from + 255) / 256, 512);
    };

    SortSource src = {tokens, nullptr, (int)V, ignore_index};
    Pair* const pairs[2] = {reinterpret_cast<Pair*>(ws + L.pairs[0]), reinterpret_cast<Pair*>(ws + L.pairs[1])};
    if (N <= (int64_t)1 << kShortBits) {
        hipLaunchKernelGGL(sort_short_kernel, dim3(1), dim3(kSortThreads), 0, s, src, pairs[0], pairs[1], N, L.share_bits, L.passes, occurs,
                           L.occurs_bytes / 16, header);
        src.pairs = pairs[(L.passes - 1) & 1];
    } else {
        uint32_t* counts = reinterpret_cast<uint32_t*>(ws + L.counts);
        const int64_t lines = (int64_t)(g.accumulate ? L.occurs : L.cleared) / 16;
        hipLaunchKernelGGL(embedding_clear_kernel, dim3((unsigned)std::min<int64_t>((lines + 255) / 256, 1024)), dim3(256), 0, s,
                           reinterpret_cast<uint4*>(ws), lines);
        hipLaunchKernelGGL(sort_count_kernel, dim3(L.blocks), dim3(kSortThreads), 0, s, src, N, (int64_t)1 << L.share_bits, counts, occurs,
                           &header->status);
        for (int pass = 0; pass < L.passes; ++pass) {
            Pair* const to = pairs[pass & 1];
            uint32_t* const later = pass + 1 < L.passes ? reinterpret_cast<uint32_t*>(ws + L.later[pass]) : nullptr;
            const int fill = take_zeros(kZerosBesidePass);
            hipLaunchKernelGGL(sort_scatter_kernel, dim3(L.blocks + fill), dim3(kSortThreads), 0, s, src, to, N, L.share_bits,
                               pass * kDigitBits, (const uint32_t*)counts, later, L.blocks, zeros);
            src.pairs = to;
            counts = later;
        }
    }
    const int slabs = slabs_of(H), waves = std::min(slabs, kSumThreads / 64);
    const unsigned columns = (unsigned)((slabs + waves - 1) / waves);
    take_zeros(V * row_bytes);
    const int64_t fill = std::min<int64_t>((zeros.upto - zeros.from + 16 * waves - 1) / (16 * waves), 4096);
    auto sums = flags & ALST_FLAG_RESIDUAL_FP32 ? run_sums_kernel<true> : run_sums_kernel<false>;
    hipLaunchKernelGGL(sums, dim3((unsigned)(L.ranges + fill), columns), dim3(waves * 64), 0, s, src.pairs, dy, N, (int)H, (int)V, L.run,
                       L.ranges, parts, g, zeros);
    if (L.ranges > 1)
        hipLaunchKernelGGL(join_kernel, dim3((unsigned)std::min(L.ranges - 1, kMostGroups), (unsigned)slabs), dim3(kJoinThreads), 0, s,
                           src.pairs, N, (int)H, (int)V, L.run, L.ranges, (const float*)parts, g);
    return hipGetLastError() == hipSuccess ? ALST_OK : ALST_ERR_HIP;
}

}  // extern "C"
