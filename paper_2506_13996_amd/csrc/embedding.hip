// Token embedding (alst_embedding.h): rows of a table by token, and the table's gradient by sorted tokens.
//
// The gradient: the row numbers are sorted by token (a stable radix sort, so that the rows of a token keep their order
// and the sums their bits), then runs of equal tokens are added up.  A wavefront takes a range of consecutive sorted rows and 512
// columns (the wavefronts of a workgroup the columns of the same rows), keeps the sum of a token's rows in registers and
// writes it out when the token changes.  Only a token of more rows than a range is cut; join_kernel adds up its partial sums.
// Rows of tokens that do not occur are filled with zeros beside the steps that leave the memory idle.
//
// Both are bound by HBM.  131072 rows of 4096 by Zipf-distributed tokens: lookup 217 us = 5.8 TB/s (245 with results written through the
// caches).  Their gradient over 128256 tokens 433 us = 4.9 TB/s (457): 36 us of sort, about 280 of sums (1.07 GB of rows in the
// tokens' order, which come at 4.5 TB/s; rows in the order of memory at 5.5), the rest zeros.  The pairs of figures below that chose
// between two forms were measured before results were written past the caches.
#include <algorithm>

#include "../../include/alst_embedding.h"
#include "rowwise.h"

namespace alst {

// ---------------------------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------------------------
constexpr int64_t kMostGroups = 1 << 22;        // workgroups of a launch (their threads have to stay below 2^32); more work is walked

constexpr int kForwardColumns = 1024;          // of a wavefront: two groups of eight values a lane
// W wavefronts (blockDim.x / 64) take ROWS rows, 1024 columns each; the R rows of wavefronts of a workgroup lie behind each other.
// A token that takes no part has no row: it is read as zeros.
template <bool F32, int ROWS, bool STREAMS>
__global__ __launch_bounds__(256) void embedding_forward_kernel(const int32_t* __restrict__ tokens, const uint16_t* __restrict__ E,
                                                                void* __restrict__ y, int64_t N, int H, int V, int ignore_index,
                                                                float scale, int32_t* __restrict__ status) {
    const uint32_t next = blockDim.x * 8, col = blockIdx.y * 2 * next + threadIdx.x * 8;
    const int64_t rows = (int64_t)blockDim.y * ROWS;
    for (int64_t g0 = blockIdx.x * rows; g0 < N; g0 += gridDim.x * rows) {
        const int64_t i0 = g0 + __builtin_amdgcn_readfirstlane(threadIdx.y) * ROWS;
        Raw8<false> r[ROWS][2];
        float factor[ROWS];                              // (0 for a row of zeros, whatever scale is)
#pragma unroll
        for (int j = 0; j < ROWS; ++j) {
            const int64_t i = i0 + j;
            const int t = __builtin_amdgcn_readfirstlane(i < N ? tokens[i] : ignore_index);
            const bool named = t >= 0 && t < V;
            if (!named && t != ignore_index && status && threadIdx.x == 0 && blockIdx.y == 0) *status = ALST_ERR_LABEL_RANGE;
            const bool kept = named && t != ignore_index;
            const RowBuffer<false> row(E, t, H, kept);
            factor[j] = kept ? scale : 0.f;
            r[j][0] = row.load(col);
            r[j][1] = row.load(col + next);
        }
#pragma unroll
        for (int j = 0; j < ROWS; ++j) {
            const RowBuffer<F32> row(y, i0 + j, H, i0 + j < N);
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float v[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = r[j][c].get(k) * factor[j];
                row.template store<STREAMS>(col + c * next, v);
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

struct EmbeddingHeader { int32_t status, joins; int32_t pad[62]; };      // joins: ranges listed for join_kernel

// Clears the marks of the tokens that occur.
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

constexpr int kZeroRows = 16;                  // of a workgroup at a time (131072 x 4096: 461 us, with 4 465, with 64 470, with 1 560)

// Rows from..upto-1 of dE without a token are filled with zeros, by workgroup `group` of `groups`.  Its wavefronts go through the
// same few rows together: a wavefront a row keeps more rows open than memory likes.
struct ZeroRows {
    void* dE;
    const uint8_t* occurs;       // [V]; NULL: every row
    int64_t from, upto;
    int halves;                  // of a row: its bytes / 2
    bool streams;
    __device__ __forceinline__ void run(int64_t group, int64_t groups) const {
        if (streams) run_as<true>(group, groups);
        else run_as<false>(group, groups);
    }
    template <bool STREAMS>
    __device__ __forceinline__ void run_as(int64_t group, int64_t groups) const {
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
        const int slabs = (halves + 511) / 512, rows = max(1, waves / slabs), mine = wave / slabs, slab = wave - mine * slabs;
        if (mine >= rows) return;
        const int step = rows == 1 ? waves : slabs;
        const float zeros[8] = {};
        for (int64_t v0 = from + group * kZeroRows; v0 < upto; v0 += groups * kZeroRows) {
            const uint64_t absent = __ballot(lane < kZeroRows && v0 + lane < upto && !(occurs && occurs[v0 + lane]));
            for (int v = mine; v < kZeroRows; v += rows) {
                if (!(absent >> v & 1)) continue;
                const RowBuffer<false> row(dE, v0 + v, halves, true);
                for (int c = slab; c < slabs; c += step) row.template store<STREAMS>(c * 512 + lane * 8, zeros);
            }
        }
    }
    int64_t groups() const { return (upto - from + kZeroRows - 1) / kZeroRows; }
};

// counts[block][digit]: the keys of a workgroup's share of the rows.  The first pass also marks the tokens that occur (unless
// NULL) and clears the status word, which its other half sets.
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(SortSource src, int64_t N, int64_t share, int shift,
                                                                  uint32_t* __restrict__ counts, uint8_t* __restrict__ occurs,
                                                                  EmbeddingHeader* header, int blocks, ZeroRows zeros) {
    __shared__ uint32_t lds[kDigits];
    if ((int)blockIdx.x >= blocks) {
        zeros.run(blockIdx.x - blocks, gridDim.x - blocks);
        return;
    }
    if (header && blockIdx.x == 0 && threadIdx.x < sizeof(EmbeddingHeader) / 4) reinterpret_cast<int32_t*>(header)[threadIdx.x] = 0;
    for (int d = threadIdx.x; d < kDigits; d += kSortThreads) lds[d] = 0;
    __syncthreads();
    const int64_t from = (int64_t)blockIdx.x * share, upto = min(from + share, N);
#pragma unroll 4
    for (int64_t i = from + threadIdx.x; i < upto; i += kSortThreads) {
        const int key = src.get(i, nullptr).key;
        atomicAdd(&lds[key >> shift & (kDigits - 1)], 1u);
        if (occurs && key < src.V) occurs[key] = 1;
    }
    __syncthreads();
    for (int d = threadIdx.x; d < kDigits; d += kSortThreads) counts[(int64_t)blockIdx.x * kDigits + d] = lds[d];
}

struct SortRoom {
    uint32_t place[kSortWaves][kDigits];      // next place of a wavefront's next key of a digit
    uint32_t sums[kSortWaves];
};

// The lanes of a wavefront with the same digit, of those that have one.
__device__ __forceinline__ uint64_t same_digit(int d, bool have) {
    uint64_t same = __ballot(have);
#pragma unroll
    for (int b = 0; b < kDigitBits; ++b) {
        const uint64_t set = __ballot(d >> b & 1);
        same &= d >> b & 1 ? set : ~set;
    }
    return same;
}

// Puts the keys of a workgroup (`block` of `blocks`) behind those of smaller digits and those of the same digit before
// them.  counts: those of all workgroups (NULL: there is one).
// A wavefront's keys are consecutive and come in batches of kBatch a lane; each finds its place among the wavefront's keys of its
// digit and, once the wavefronts' numbers are added up, among all.  A share of one batch a wavefront stays in registers
// between the two, a longer one is read again.
__device__ __forceinline__ void sort_scatter(const SortSource& src, Pair* __restrict__ to, int64_t N, int share_bits, int shift,
                                             const uint32_t* __restrict__ counts, int block, int blocks, SortRoom& room,
                                             int32_t* status) {
    constexpr int kBatch = 4;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int d = threadIdx.x; d < kSortWaves * kDigits; d += kSortThreads) (&room.place[0][0])[d] = 0;
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
    const int64_t share = (int64_t)1 << share_bits, each = share / kSortWaves;
    const int64_t from = min(block * share + wave * each, N), upto = min(from + each, N);
    const bool one = each == 64 * kBatch;
    volatile uint32_t* const mine = room.place[wave];
    Pair p[kBatch];
    uint32_t place[kBatch];
    auto batch = [&](int64_t i0, int32_t* said) {          // reads the batch and places it behind the wavefront's keys so far
#pragma unroll
        for (int j = 0; j < kBatch; ++j) p[j] = i0 + j * 64 + lane < upto ? src.get(i0 + j * 64 + lane, said) : Pair{0, 0};
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const bool have = i0 + j * 64 + lane < upto;
            const int d = (p[j].key >> shift) & (kDigits - 1);
            const uint64_t same = same_digit(d, have);
            const int rank = __popcll(same & (((uint64_t)1 << lane) - 1));
            place[j] = have ? mine[d] + rank : 0;
            __builtin_amdgcn_wave_barrier();
            if (have && rank == 0) mine[d] = place[j] + __popcll(same);
            __builtin_amdgcn_wave_barrier();
        }
    };
    for (int64_t i0 = from; i0 < upto; i0 += 64 * kBatch) batch(i0, status);
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
    auto put = [&](int64_t i0, bool placed) {
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            if (i0 + j * 64 + lane >= upto) continue;
            const uint32_t at = place[j] + (placed ? 0u : mine[(p[j].key >> shift) & (kDigits - 1)]);
            to[at] = p[j];
        }
    };
    if (one) {
        put(from, false);
    } else {
        for (int64_t i0 = from; i0 < upto; i0 += 64 * kBatch) {      // (this time the places count on from the first of all)
            batch(i0, nullptr);
            put(i0, true);
        }
    }
}

// A pass, and beside it (workgroups from `blocks` on) rows of zeros.
__global__ __launch_bounds__(kSortThreads) void sort_scatter_kernel(SortSource src, Pair* __restrict__ to, int64_t N, int share_bits,
                                                                    int shift, const uint32_t* __restrict__ counts, int blocks,
                                                                    int32_t* status, ZeroRows zeros) {
    __shared__ SortRoom room;
    if ((int)blockIdx.x >= blocks) {
        zeros.run(blockIdx.x - blocks, gridDim.x - blocks);
        return;
    }
    sort_scatter(src, to, N, share_bits, shift, counts, blockIdx.x, blocks, room, status);
}

// All of the sort where one workgroup's share holds the rows.  Beside it (the other workgroups) every row is filled with zeros:
// so few tokens leave most of them that way.
__global__ __launch_bounds__(kSortThreads) void sort_short_kernel(SortSource src, Pair* a, Pair* b, int64_t N, int share_bits, int passes,
                                                                  EmbeddingHeader* header, ZeroRows zeros) {
    __shared__ SortRoom room;
    if (blockIdx.x > 0) {
        zeros.run(blockIdx.x - 1, gridDim.x - 1);
        return;
    }
    if (threadIdx.x < sizeof(EmbeddingHeader) / 4) reinterpret_cast<int32_t*>(header)[threadIdx.x] = 0;
    __syncthreads();
    for (int pass = 0; pass < passes; ++pass) {
        sort_scatter(src, pass & 1 ? b : a, N, share_bits, pass * kDigitBits, nullptr, 0, 1, room, pass ? nullptr : &header->status);
        src.pairs = pass & 1 ? b : a;
        __threadfence_block();
        __syncthreads();
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

template <bool F32, bool STREAMS>
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
    row.template store<STREAMS>(col, v);
}
template <bool STREAMS>
__device__ __forceinline__ void write_grad(const Grad& g, int key, int H, uint32_t col, const float (&sum)[8]) {
    if (g.f32) write_grad_as<true, false>(g, key, H, col, sum);
    else write_grad_as<false, STREAMS>(g, key, H, col, sum);
}

constexpr int kSumThreads = 512;
template <bool F32> constexpr int kRowsTogether = F32 ? 8 : 16;      // rows of dy that a wavefront has in flight (459 us; 465 with 8)
constexpr int kJoinThreads = 512;
constexpr int kJoinGroups = 256;               // workgroups of the joins' launch for each 512 columns, which walk the list

// A range is `run` sorted rows.  Its wavefronts add up the tokens that begin in it, and follow the last one into the next range.
// Only a token that goes through a whole range besides is cut: parts[range][1] has its rows of the range where it begins, which is
// then listed, parts[range][0] those of the ranges behind.  A workgroup: a range and 512 columns a wavefront; workgroups from
// `ranges` on: rows of zeros.
template <bool F32, bool STREAMS>
__global__ __launch_bounds__(kSumThreads) void run_sums_kernel(const Pair* __restrict__ pairs, const void* __restrict__ dy, int64_t N,
                                                               int H, int V, int run, int64_t ranges, float* __restrict__ parts,
                                                               Pair* __restrict__ list, EmbeddingHeader* header, Grad g, ZeroRows zeros) {
    constexpr int kTogether = kRowsTogether<F32>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int64_t range = blockIdx.x, p0 = range * run;
    if (range >= ranges) {
        zeros.run((range - ranges) * gridDim.y + blockIdx.y, (gridDim.x - ranges) * gridDim.y);
        return;
    }
    const uint32_t col = (blockIdx.y * waves + wave) * 512 + lane * 8;
    const int64_t end = min(p0 + run, N);
    // keys next to the borders of this range, of the one before and of the one behind (V: no row there)
    auto key_at = [&](int64_t i) { return __builtin_amdgcn_readfirstlane(i >= 0 && i < N ? pairs[i].key : V); };
    const int first = key_at(p0), last = key_at(end - 1), next = key_at(end);
    if (first >= V) return;
    const bool came = p0 > 0 && key_at(p0 - 1) == first, goes_on = next == last && last < V, through = came && goes_on && first == last;
    const bool head_cut = came && (through || (p0 > run && key_at(p0 - run - 1) == first));
    const bool tail_cut = goes_on && !through && key_at(p0 + 2 * run) == last;
    // rows from `start` to `stop`: without those of a token that the range before takes, with those of one that ends in the next
    auto length = [&](int64_t from, int key) {           // rows with `key`, of the run rows from `from`
        int n = 0;
        for (int b = 0; b < run; b += 64) n += __popcll(__ballot(b + lane < run && from + b + lane < N && pairs[from + b + lane].key == key));
        return n;
    };
    const int64_t start = came && !head_cut ? p0 + length(p0, first) : p0;
    const int64_t stop = goes_on && !through && !tail_cut ? end + length(end, last) : end;
    float sum[8] = {};
    bool head = head_cut;
    for (int64_t b0 = start; b0 < stop; b0 += 64) {      // 64 rows, whose pairs the lanes hold
        Pair mine = {V, 0};
        if (b0 + lane < stop) mine = pairs[b0 + lane];
        const int here = (int)min((int64_t)64, stop - b0);
        const int follows = b0 + 64 < stop ? key_at(b0 + 64) : -1;
        for (int j0 = 0; j0 < here; j0 += kTogether) {
            Raw8<F32> r[kTogether];
#pragma unroll
            for (int j = 0; j < kTogether; ++j) {
                const int key = __builtin_amdgcn_readlane(mine.key, j0 + j), row = __builtin_amdgcn_readlane(mine.row, j0 + j);
                r[j] = RowBuffer<F32>(dy, row, H, key < V).load(col);
            }
#pragma unroll
            for (int j = 0; j < kTogether; ++j) {
                const int at = j0 + j;
                const int key = __builtin_amdgcn_readlane(mine.key, at);
                if (key >= V) return;                    // (no rows behind the last token's, or behind `stop`)
#pragma unroll
                for (int k = 0; k < 8; ++k) sum[k] += r[j].get(k);
                if (key == (at + 1 == here ? follows : __builtin_amdgcn_readlane(mine.key, (at + 1) & 63))) continue;
                if (head) {
                    RowBuffer<true>(parts, range * 2, H, true).store(col, sum);
                } else if (tail_cut && b0 + at + 1 == stop) {
                    RowBuffer<true>(parts, range * 2 + 1, H, true).store(col, sum);
                    if (blockIdx.y == 0 && threadIdx.x == 0) list[atomicAdd(&header->joins, 1)] = {key, (int32_t)range};
                } else {
                    write_grad<STREAMS>(g, key, H, col, sum);
                }
                head = false;
#pragma unroll
                for (int k = 0; k < 8; ++k) sum[k] = 0.f;
            }
        }
    }
}

// The tokens that were cut: the partial sums of the range where one begins (slot 1) and of those behind it (slot 0), dealt to the
// wavefronts of the workgroup in turn.  The list's order changes nothing: each token has its own row.  The first `groups` workgroups
// walk the list, 512 columns each, and wait for memory most of their time (18 us); the others fill rows with zeros beside them.
__global__ __launch_bounds__(kJoinThreads) void join_kernel(const Pair* __restrict__ pairs, int64_t N, int H, int run, int64_t ranges,
                                                            int slabs, int groups, const Pair* __restrict__ list,
                                                            const EmbeddingHeader* __restrict__ header, const float* __restrict__ parts,
                                                            Grad g, ZeroRows zeros) {
    constexpr int kWaves = kJoinThreads / 64;
    __shared__ float lds[kWaves][512];
    if ((int)blockIdx.x >= groups) {
        zeros.run(blockIdx.x - groups, gridDim.x - groups);
        return;
    }
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int slab = blockIdx.x % slabs, step = groups / slabs;
    const uint32_t col = slab * 512 + lane * 8;
    // (the first entry is asked for with their number; the list has room for `step` entries at least)
    int item = blockIdx.x / slabs;
    Pair entry = list[item];
    const int joins = header->joins;
    for (; item < joins; item += step) {
        if (item >= step) entry = list[item];
        const int64_t range = __builtin_amdgcn_readfirstlane(entry.row);
        const int key = __builtin_amdgcn_readfirstlane(entry.key);
        int64_t more = 0;                                    // ranges behind that begin with it
        for (int n = kJoinThreads; n == kJoinThreads; more += n) {
            const int64_t r = range + 1 + more + threadIdx.x;
            n = __syncthreads_count(r < ranges && pairs[r * run].key == key);
        }
        float sum[8] = {};
        auto add = [&](int64_t first, int64_t step) {      // eight of them in flight
            for (int64_t k = first; k <= more; k += 8 * step) {
                Raw8<true> r[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int64_t at = k + j * step;
                    r[j] = RowBuffer<true>(parts, (range + at) * 2 + (at == 0), H, at <= more).load(col);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum[i] += r[j].get(i);
            }
        };
        add(wave, kWaves);
        if (wave != 0) store8(lds[wave], lane * 8, sum);
        __syncthreads();
        if (wave == 0) {
#pragma unroll
            for (int w = 1; w < kWaves; ++w) {
                const Raw8<true> r = load8(lds[w], lane * 8);
#pragma unroll
                for (int j = 0; j < 8; ++j) sum[j] += r.get(j);
            }
            write_grad<false>(g, key, H, col, sum);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------------
constexpr int kMostRun = 128;
// Zeros beside a pass of the sort that moves rows (12 us) and beside the joins (18 us): about what the memory takes in that time, which
// hardly goes by N and H.  Beside a pass, 64 MB against none / 32 / 128: 131072 x 4096 of 128256 434 us against 443 / 440 / 432, 8192 x
// 8192 of 128256 446 against 460 / 450 / 440, 16384 x 1600 of 50257 57 against 65 / 59 / 65; narrow rows lose, 300000 x 256 of 200000 114
// against 109 / 109 / 113.  Beside the joins, 96 MB against none / 48 / 192: the first 434 against 436 / 434 / 438, the second 446
// against 448 / 446 / 443, the others the same.
constexpr int64_t kZerosBesidePass = (int64_t)64 << 20, kZerosBesideJoins = (int64_t)96 << 20;
constexpr int kShortBits = 12;                 // up to 4096 rows are sorted by one workgroup, beside zeros for every row (3001 x 1600 of
                                               // 50257: 42 us; 51 when the zeros wait for the marks of the sorted tokens)

struct EmbeddingLayout {
    int share_bits;              // rows of a workgroup of the sort: 2^share_bits
    int blocks, passes, run;
    int64_t ranges, occurs_bytes;
    size_t counts, occurs, pairs[2], list, parts, total;       // behind the header
};

static int slabs_of(int64_t H) { return (int)((H + 511) / 512); }

// Sorted rows of a range: kMostRun (131072 x 4096: 459 us, with 64 474 and with 256 500), fewer where that leaves less than 4096
// wavefronts.
static int run_of(int64_t N, int64_t H) {
    int run = kMostRun;
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
    L.counts = take((size_t)kMostSortBlocks * kDigits * 4);
    L.occurs = take((size_t)V);
    L.occurs_bytes = (int64_t)(o - L.occurs);
    L.pairs[0] = take((size_t)N * sizeof(Pair));
    L.pairs[1] = take((size_t)N * sizeof(Pair));
    // (runs get longer with N: room for the partial sums of every shorter call)
    int64_t ranges = 0;
    for (int run = 8; run <= L.run; run *= 2) {
        const int64_t most = run < kMostRun ? std::min(N, ((int64_t)run * 2 * 4096 - 1) / slabs_of(H)) : N;
        ranges = std::max(ranges, (most + run - 1) / run);
    }
    L.list = take((size_t)ranges * sizeof(Pair));
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
    if (H % 8 != 0 || !aligned_to(tokens, 4) || !aligned_to(E, 16) || !aligned_to(y, 16) || !aligned_to(device_status_out, 4))
        return ALST_ERR_ALIGN;
    const int W = (int)std::min<int64_t>((H + kForwardColumns - 1) / kForwardColumns, 4), R = 4 / W;
    // a row a wavefront at a time (131072 x 4096: 245 us, 262 with four); of short rows four, or the launch waits for tokens
    // (262144 x 64: 32 us, 47 with one)
    const int together = W == 1 ? 4 : 1;
    const int64_t rows = (int64_t)R * together, columns = (int64_t)W * kForwardColumns;
    const dim3 grid((unsigned)std::min((N + rows - 1) / rows, kMostGroups), (unsigned)((H + columns - 1) / columns));
    const bool f32 = flags & ALST_FLAG_RESIDUAL_FP32;
    const bool streams = streams_out(N * H * 2);
    auto kernel = together == 1 ? (f32       ? embedding_forward_kernel<true, 1, false>
                                   : streams ? embedding_forward_kernel<false, 1, true>
                                             : embedding_forward_kernel<false, 1, false>)
                                : (f32       ? embedding_forward_kernel<true, 4, false>
                                   : streams ? embedding_forward_kernel<false, 4, true>
                                             : embedding_forward_kernel<false, 4, false>);
    hipLaunchKernelGGL(kernel, grid, dim3(W * 64, R), 0, (hipStream_t)stream, tokens, (const uint16_t*)E, y, N, (int)H, (int)V,
                       ignore_index, scale, device_status_out);
    return hipGetLastError() == hipSuccess ? ALST_OK : ALST_ERR_HIP;
}

int alst_embedding_backward(const int32_t* tokens, const void* dy, int64_t N, int64_t H, int64_t V, int32_t ignore_index, float scale,
                            void* dE, void* workspace, size_t workspace_bytes, uint32_t flags, void* stream) {
    if (!tokens || !dy || !dE || !workspace) return ALST_ERR_NULL;
    if (flags & ~(ALST_FLAG_RESIDUAL_FP32 | ALST_FLAG_DW_FP32 | ALST_FLAG_DW_ACCUMULATE)) return ALST_ERR_UNSUPPORTED;
    if (!embedding_shape_ok(N, H, V)) return ALST_ERR_SHAPE;
    if (H % 8 != 0 || !aligned_to(tokens, 4) || !aligned_to(dy, 16) || !aligned_to(dE, 16) || !aligned_to(workspace, 16))
        return ALST_ERR_ALIGN;
    const EmbeddingLayout L = make_embedding_layout(N, H, V);
    if (workspace_bytes < L.total) return ALST_ERR_WORKSPACE;
    const hipStream_t s = (hipStream_t)stream;
    unsigned char* const ws = static_cast<unsigned char*>(workspace);
    EmbeddingHeader* const header = reinterpret_cast<EmbeddingHeader*>(ws);
    float* const parts = reinterpret_cast<float*>(ws + L.parts);
    const bool sums32 = flags & ALST_FLAG_DW_FP32;
    const int64_t row_bytes = H * (sums32 ? 4 : 2);
    const Grad g = {dE, scale, sums32, (flags & ALST_FLAG_DW_ACCUMULATE) != 0};
    const bool streams = streams_out(V * row_bytes);
    uint8_t* const occurs = g.accumulate ? nullptr : ws + L.occurs;
    // rows of zeros: a share beside each step of the sort (whose few workgroups leave the memory idle for about that many bytes'
    // time), the rest beside the sums
    ZeroRows zeros = {dE, occurs, 0, 0, (int)(row_bytes / 2), streams};
    auto take_zeros = [&](int64_t bytes) {               // workgroups of 16 wavefronts that fill the next `bytes`
        zeros.from = zeros.upto;
        if (g.accumulate || bytes == 0) return 0;
        zeros.upto = std::min<int64_t>(V, zeros.from + (bytes + row_bytes - 1) / row_bytes);
        return (int)std::min<int64_t>(zeros.groups(), 2048);
    };

    SortSource src = {tokens, nullptr, (int)V, ignore_index};
    Pair* const pairs[2] = {reinterpret_cast<Pair*>(ws + L.pairs[0]), reinterpret_cast<Pair*>(ws + L.pairs[1])};
    if (N <= (int64_t)1 << kShortBits) {
        zeros.occurs = nullptr;
        const int fill = take_zeros(V * row_bytes);
        hipLaunchKernelGGL(sort_short_kernel, dim3(1 + fill), dim3(kSortThreads), 0, s, src, pairs[0], pairs[1], N, L.share_bits, L.passes,
                           header, zeros);
        src.pairs = pairs[(L.passes - 1) & 1];
    } else {
        uint32_t* const counts = reinterpret_cast<uint32_t*>(ws + L.counts);
        const int64_t lines = L.occurs_bytes / 16;
        if (occurs)
            hipLaunchKernelGGL(embedding_clear_kernel, dim3((unsigned)std::min<int64_t>((lines + 255) / 256, 1024)), dim3(256), 0, s,
                               reinterpret_cast<uint4*>(occurs), lines);
        for (int pass = 0; pass < L.passes; ++pass) {
            Pair* const to = pairs[pass & 1];
            const int shift = pass * kDigitBits;
            int fill = pass ? take_zeros(kZerosBesidePass / 2) : 0;       // (the first one makes the marks)
            hipLaunchKernelGGL(sort_count_kernel, dim3(L.blocks + fill), dim3(kSortThreads), 0, s, src, N, (int64_t)1 << L.share_bits, shift,
                               counts, pass ? nullptr : occurs, pass ? nullptr : header, L.blocks, zeros);
            fill = take_zeros(kZerosBesidePass);
            hipLaunchKernelGGL(sort_scatter_kernel, dim3(L.blocks + fill), dim3(kSortThreads), 0, s, src, to, N, L.share_bits, shift,
                               (const uint32_t*)counts, L.blocks, pass ? nullptr : &header->status, zeros);
            src.pairs = to;
        }
    }
    const int slabs = slabs_of(H), most = kSumThreads / 64, columns = (slabs + most - 1) / most, waves = (slabs + columns - 1) / columns;
    const int64_t left = (V - zeros.upto) * row_bytes;
    const bool join = L.ranges > 2;                      // (a token that is cut has three ranges at least)
    take_zeros(join ? std::max<int64_t>(left - kZerosBesideJoins, 0) : left);
    const int64_t fill = std::min((zeros.groups() + columns - 1) / columns, kMostGroups);
    Pair* const list = reinterpret_cast<Pair*>(ws + L.list);
    auto sums = flags & ALST_FLAG_RESIDUAL_FP32 ? (streams ? run_sums_kernel<true, true> : run_sums_kernel<true, false>)
                                                : (streams ? run_sums_kernel<false, true> : run_sums_kernel<false, false>);
    hipLaunchKernelGGL(sums, dim3((unsigned)(L.ranges + fill), (unsigned)columns), dim3(waves * 64), 0, s, src.pairs, dy, N, (int)H, (int)V,
                       L.run, L.ranges, parts, list, header, g, zeros);
    if (join) {
        const int fill_join = take_zeros(left), groups = (int)std::min<int64_t>(L.ranges / 2, kJoinGroups) * slabs;
        hipLaunchKernelGGL(join_kernel, dim3(groups + fill_join), dim3(kJoinThreads), 0, s, src.pairs, N, (int)H, L.run, L.ranges, slabs, groups,
                           (const Pair*)list, (const EmbeddingHeader*)header, (const float*)parts, g, zeros);
    }
    return hipGetLastError() == hipSuccess ? ALST_OK : ALST_ERR_HIP;
}

}  // extern "C"
