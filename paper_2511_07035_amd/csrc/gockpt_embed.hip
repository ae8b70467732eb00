// gockpt_embed.hip -- embedding lookup with scaling, and its gradient.
//
//   lookup_kernel  out[t] = round(scale * table[id[t]]), zeros for masked ids.
//
//   The gradient of row v is scale * (sum of grad_out over the tokens with id
//   v).  The table's rows are cut into buckets of 2^b rows (64, more for large
//   tables); a bucket's tokens are found, sorted by (row, token), and summed
//   row by row in registers.  No atomics on sums, so the same bits every time.
//   Few tokens: every bucket's blocks look through all ids (rows_kernel<..., true>).
//   Many tokens: count_kernel and place_kernel bring the tokens into bucket
//   order first (stable: token order within a bucket), rows_kernel takes each
//   bucket, or each chunk of kChunk tokens of a larger one, whose fp32 sums
//   join_kernel adds in chunk order.
#include <limits.h>

#include "gockpt_ops_internal.h"

#pragma clang fp contract(off)

namespace gockpt {

namespace {

constexpr int kThreads = 256;
constexpr int kVecCols = 8;  // columns of a lane

// Eight consecutive elements, and fewer at a row's end.
template <int kT>
struct Raw {
    u32x4 w[kT == kFP32 ? 2 : 1];
};

// Columns c to c + 7 of the row at p, zeros from `cols` on.
template <int kT>
__device__ __forceinline__ Raw<kT> load8(const uint8_t* p, int64_t c, int64_t cols) {
    constexpr int kB = kT == kFP32 ? 4 : 2;
    Raw<kT> r;
    p += c * kB;
    if (c + kVecCols <= cols) {
        r.w[0] = *reinterpret_cast<const u32x4_any*>(p);
        if constexpr (kT == kFP32) r.w[1] = *reinterpret_cast<const u32x4_any*>(p + 16);
    } else {
        uint32_t e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            e[i] = 0u;
            if (c + i < cols) {
                if constexpr (kT == kFP32)
                    e[i] = reinterpret_cast<const uint32_t*>(p)[i];
                else
                    e[i] = reinterpret_cast<const uint16_t*>(p)[i];
            }
        }
        if constexpr (kT == kFP32) {
            r.w[0] = (u32x4){e[0], e[1], e[2], e[3]};
            r.w[1] = (u32x4){e[4], e[5], e[6], e[7]};
        } else {
            r.w[0] = (u32x4){e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16};
        }
    }
    return r;
}

template <int kT>
__device__ __forceinline__ void widen8(const Raw<kT>& r, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (kT == kFP32)
            x[i] = __uint_as_float(r.w[i / 4][i % 4]);
        else
            x[i] = elem_to_f32<kT>(r.w[0][i / 2] >> (16 * (i % 2)) & 0xFFFFu);
    }
}

template <int kT>
__device__ __forceinline__ void store8(uint8_t* p, int64_t c, int64_t cols, const float (&x)[8]) {
    constexpr int kB = kT == kFP32 ? 4 : 2;
    p += c * kB;
    if (c + kVecCols <= cols) {
        if constexpr (kT == kFP32) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
                *reinterpret_cast<u32x4_any*>(p + 16 * h) =
                    (u32x4){__float_as_uint(x[4 * h]), __float_as_uint(x[4 * h + 1]), __float_as_uint(x[4 * h + 2]),
                            __float_as_uint(x[4 * h + 3])};
        } else {
            *reinterpret_cast<u32x4_any*>(p) =
                (u32x4){pack2<kT>(x[0], x[1]), pack2<kT>(x[2], x[3]), pack2<kT>(x[4], x[5]), pack2<kT>(x[6], x[7])};
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < cols) store_elem<kT>(p + kB * i, x[i]);
    }
}

struct Ids {
    const void* p;
    int64_t stride, first;
    int64_t padding;   // id that adds nothing to a gradient
    uint32_t tokens, length;
    int32_t wide;      // 64-bit ids
    uint32_t rows;     // of the table, at most INT32_MAX
};

// Row of token t (t < tokens), or -1 where it is masked.
__device__ __forceinline__ int32_t token_row(const Ids& ids, uint32_t t, bool grad) {
    int64_t at = t;
    if (ids.stride != ids.length) {
        const uint32_t b = t / ids.length;
        at = b * ids.stride + (t - b * ids.length);
    }
    const int64_t id = ids.wide ? static_cast<const int64_t*>(ids.p)[at] : static_cast<const int32_t*>(ids.p)[at];
    // as unsigned, so that no id overflows
    const uint64_t r = static_cast<uint64_t>(id) - static_cast<uint64_t>(ids.first);
    if (r >= ids.rows || id < ids.first || (grad && id == ids.padding)) return -1;
    return static_cast<int32_t>(r);
}

// ---- lookup ------------------------------------------------------------------

struct LookupArgs {
    Ids ids;
    const uint8_t* table;
    uint8_t* out;
    int64_t cols, table_stride, out_stride;  // strides in bytes
    float scale;
    int32_t lanes;  // lanes of a row, a power of two
};

constexpr int kLookupRows = 4;  // rows of a thread

// A block takes kThreads / lanes rows at a time, kLookupRows times, and the
// columns blockIdx.y * lanes * 8 on.
template <int kW, int kO>
__global__ __launch_bounds__(kThreads) void lookup_kernel(LookupArgs a) {
    const uint32_t lane = threadIdx.x & (a.lanes - 1);
    const uint32_t per = kThreads / a.lanes;
    const int64_t c = (static_cast<int64_t>(blockIdx.y) * a.lanes + lane) * kVecCols;
    if (c >= a.cols) return;
    const uint32_t t0 = blockIdx.x * per * kLookupRows + threadIdx.x / a.lanes;
    int32_t row[kLookupRows];
#pragma unroll
    for (int i = 0; i < kLookupRows; ++i) {
        const uint32_t t = t0 + i * per;
        row[i] = t < a.ids.tokens ? token_row(a.ids, t, false) : -1;
    }
    Raw<kW> raw[kLookupRows];
#pragma unroll
    for (int i = 0; i < kLookupRows; ++i) {
        raw[i] = Raw<kW>{};
        if (row[i] >= 0) raw[i] = load8<kW>(a.table + row[i] * a.table_stride, c, a.cols);
    }
#pragma unroll
    for (int i = 0; i < kLookupRows; ++i) {
        const uint32_t t = t0 + i * per;
        if (t >= a.ids.tokens) continue;
        float x[8];
        widen8<kW>(raw[i], x);
        // a masked token's zeros stay +0 whatever the scale
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = row[i] >= 0 ? x[k] * a.scale : 0.0f;
        store8<kO>(a.out + t * a.out_stride, c, a.cols, x);
    }
}

// ---- gradient ----------------------------------------------------------------

constexpr int kMinBucketBits = 6;   // 64 rows
constexpr int kMaxBucketBits = 10;
constexpr int kMaxBuckets = 4096;
constexpr int kChunk = 512;         // tokens of a bucket that one block sums
constexpr int kDirectTokens = 2048; // up to these every block looks through all ids
constexpr int kPlaceThreads = 1024;
constexpr int kPlaceWaves = kPlaceThreads / 64;
constexpr int kMaxPlaceBlocks = 64;
constexpr int kAhead = 8;           // tokens whose loads are in flight

struct Item {
    int32_t bucket, first, count, pad;
};
struct Split {
    int32_t bucket, item, count, pad;  // its chunks: items item to item + count - 1
};

struct GradArgs {
    Ids ids;
    const uint8_t* src;
    uint8_t* dst;
    int64_t cols, src_stride, dst_stride;  // strides in bytes
    float scale;
    int32_t dst_dtype, accumulate;
    int32_t lanes;
    int32_t bits, buckets;                 // rows of a bucket: 1 << bits
    int32_t place_blocks, place_tokens;    // tokens of a place block, a multiple of kPlaceThreads
    int32_t max_items, max_splits;
    // workspace
    uint32_t* counts;    // [place_blocks][buckets]
    uint32_t* starts;    // [buckets + 1]
    int32_t* heads;      // items, splits
    Item* items;
    Split* splits;
    u32x2* sorted;       // {row within the bucket, token}
    uint8_t* present;    // [max_items][rows of a bucket]
    float* partial;      // [max_items][rows of a bucket][cols rounded up to 8]
};

__global__ __launch_bounds__(kPlaceThreads) void count_kernel(GradArgs a) {
    __shared__ uint32_t n[kMaxBuckets];
    for (int j = threadIdx.x; j < a.buckets; j += kPlaceThreads) n[j] = 0u;
    __syncthreads();
    const uint32_t t0 = blockIdx.x * static_cast<uint32_t>(a.place_tokens);
    for (int i = threadIdx.x; i < a.place_tokens; i += kPlaceThreads) {
        const int32_t row = t0 + i < a.ids.tokens ? token_row(a.ids, t0 + i, true) : -1;
        if (row >= 0) atomicAdd(&n[row >> a.bits], 1u);
    }
    __syncthreads();
    for (int j = threadIdx.x; j < a.buckets; j += kPlaceThreads) a.counts[blockIdx.x * a.buckets + j] = n[j];
}

// Exclusive prefix sum of x over the block's threads; total gets the sum.
__device__ __forceinline__ uint64_t block_scan(uint64_t x, uint64_t& total) {
    __shared__ uint64_t wave[kPlaceWaves];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    uint64_t s = x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint64_t y = __shfl_up(s, o, 64);
        if (lane >= o) s += y;
    }
    __syncthreads();
    if (lane == 63) wave[w] = s;
    __syncthreads();
    uint64_t before = 0;
    total = 0;
    for (int i = 0; i < kPlaceWaves; ++i) {
        if (i < w) before += wave[i];
        total += wave[i];
    }
    return before + s - x;
}

// Writes the block's tokens to their places in bucket order; block 0 also the
// buckets' starts and the table of the chunks of those larger than kChunk.
__global__ __launch_bounds__(kPlaceThreads) void place_kernel(GradArgs a) {
    __shared__ uint32_t place[kMaxBuckets];              // next place of each bucket for this block
    __shared__ uint8_t in_wave[kPlaceWaves][kMaxBuckets];  // tokens of each bucket in each wavefront's 64
    constexpr int kPer = kMaxBuckets / kPlaceThreads;
    const int j0 = threadIdx.x * kPer;
    uint32_t total[kPer], before[kPer];
    uint64_t mine = 0, all;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        total[i] = before[i] = 0u;
        if (j0 + i < a.buckets) {
            for (int b = 0; b < a.place_blocks; ++b) {
                const uint32_t n = a.counts[b * a.buckets + j0 + i];
                if (b < static_cast<int>(blockIdx.x)) before[i] += n;
                total[i] += n;
            }
        }
        mine += total[i];
    }
    uint64_t start = block_scan(mine, all);
    uint64_t split = 0;  // chunks in the low half, split buckets in the high half
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        if (j0 + i < a.buckets) {
            place[j0 + i] = static_cast<uint32_t>(start) + before[i];
            if (blockIdx.x == 0) a.starts[j0 + i] = static_cast<uint32_t>(start);
        }
        start += total[i];
        if (total[i] > kChunk) split += (total[i] + kChunk - 1) / kChunk + (uint64_t{1} << 32);
    }
    if (blockIdx.x == 0) {
        uint64_t at = block_scan(split, split);
        if (threadIdx.x == 0) {
            a.starts[a.buckets] = static_cast<uint32_t>(all);
            a.heads[0] = static_cast<int32_t>(split & 0xFFFFFFFFu);
            a.heads[1] = static_cast<int32_t>(split >> 32);
        }
        uint32_t first = static_cast<uint32_t>(start);
#pragma unroll
        for (int i = kPer - 1; i >= 0; --i) first -= total[i];
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if (total[i] > kChunk) {
                const int n = static_cast<int>((total[i] + kChunk - 1) / kChunk);
                const int item = static_cast<int>(at & 0xFFFFFFFFu);
                a.splits[at >> 32] = {j0 + i, item, n, 0};
                for (int k = 0; k < n; ++k) {
                    const uint32_t left = total[i] - k * kChunk;
                    a.items[item + k] = {j0 + i, static_cast<int32_t>(first + k * kChunk),
                                         static_cast<int32_t>(left < kChunk ? left : kChunk), 0};
                }
                at += n + (uint64_t{1} << 32);
            }
            first += total[i];
        }
    }
    for (int j = threadIdx.x; j < a.buckets; j += kPlaceThreads)
#pragma unroll
        for (int w = 0; w < kPlaceWaves; ++w) in_wave[w][j] = 0;
    __syncthreads();

    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const uint32_t t0 = blockIdx.x * static_cast<uint32_t>(a.place_tokens);
    for (int i = 0; i < a.place_tokens; i += kPlaceThreads) {
        const uint32_t t = t0 + i + threadIdx.x;
        const int32_t row = t < a.ids.tokens ? token_row(a.ids, t, true) : -1;
        const uint32_t bucket = row >= 0 ? static_cast<uint32_t>(row) >> a.bits : 0u;
        // the lanes of this wavefront with the same bucket
        uint64_t same = __ballot(row >= 0);
        for (int b = 0; (a.buckets - 1) >> b; ++b) {
            const bool bit = bucket >> b & 1u;
            const uint64_t m = __ballot(bit);
            same &= bit ? m : ~m;
        }
        const int rank = __popcll(same & ((uint64_t{1} << lane) - 1));
        const bool leads = row >= 0 && rank == 0;
        if (leads) in_wave[w][bucket] = static_cast<uint8_t>(__popcll(same));
        __syncthreads();
        if (row >= 0) {
            uint32_t at = place[bucket] + rank;
            for (int k = 0; k < w; ++k) at += in_wave[k][bucket];
            a.sorted[at] = (u32x2){static_cast<uint32_t>(row) & ((1u << a.bits) - 1u), t};
        }
        __syncthreads();
        if (leads) {
            atomicAdd(&place[bucket], static_cast<uint32_t>(__popcll(same)));
            in_wave[w][bucket] = 0;
        }
        __syncthreads();
    }
}

template <int kD>
__device__ __forceinline__ void finish_row(const GradArgs& a, int64_t row, int64_t c, const float (&acc)[8],
                                           bool add) {
    uint8_t* p = a.dst + row * a.dst_stride;
    float x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = acc[k] * a.scale;
    if (add) {
        float old[8];
        widen8<kD>(load8<kD>(p, c, a.cols), old);
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = old[k] + x[k];
    }
    store8<kD>(p, c, a.cols, x);
}

__device__ __forceinline__ void finish_row(const GradArgs& a, int64_t row, int64_t c, const float (&acc)[8],
                                           bool add) {
    if (a.dst_dtype == kBF16)
        finish_row<kBF16>(a, row, c, acc, add);
    else if (a.dst_dtype == kFP16)
        finish_row<kFP16>(a, row, c, acc, add);
    else
        finish_row<kFP32>(a, row, c, acc, add);
}

// One bucket's tokens, or one chunk of them: sorted by (row, token) in LDS by
// counting, for each, the smaller keys; then summed row by row.  A row is
// `lanes` lanes wide, the block's groups of so many lanes take equal ranges of
// rows, and blockIdx.y goes over the columns.
template <int kS, bool kDirect>
__global__ __launch_bounds__(kThreads) void rows_kernel(GradArgs a) {
    constexpr int kCap = kDirect ? kDirectTokens : kChunk;
    __shared__ alignas(16) uint32_t key[kCap + 4];  // row << 16 | place in the list (or the token)
    __shared__ uint32_t tok[kDirect ? 1 : kCap];
    __shared__ uint32_t by_row[kCap];    // tokens in order
    __shared__ uint16_t row_of[kCap];
    __shared__ uint32_t seen[(1 << kMaxBucketBits) / 32];
    __shared__ uint32_t group_end[kThreads];
    __shared__ uint32_t count;

    const int rows = 1 << a.bits;
    int bucket, n = 0, first = 0, item = -1;
    if constexpr (kDirect) {
        bucket = blockIdx.x;
    } else if (static_cast<int>(blockIdx.x) < a.max_items) {
        if (static_cast<int>(blockIdx.x) >= a.heads[0]) return;
        item = blockIdx.x;
        const Item it = a.items[item];
        bucket = it.bucket;
        first = it.first;
        n = it.count;
    } else {
        bucket = blockIdx.x - a.max_items;
        first = a.starts[bucket];
        n = static_cast<int>(a.starts[bucket + 1]) - first;
        if (n > kChunk) return;  // its chunks are items
        if (n == 0 && a.accumulate) return;
    }
    if (threadIdx.x < rows / 32) seen[threadIdx.x] = 0u;
    group_end[threadIdx.x] = 0u;
    if constexpr (kDirect) {
        if (threadIdx.x == 0) count = 0u;
        __syncthreads();
        for (uint32_t t = threadIdx.x; t < a.ids.tokens; t += kThreads) {
            const int32_t row = token_row(a.ids, t, true);
            if (row >= 0 && row >> a.bits == bucket)
                key[atomicAdd(&count, 1u)] = static_cast<uint32_t>(row & (rows - 1)) << 16 | t;
        }
        __syncthreads();
        n = static_cast<int>(count);
        if (n == 0 && a.accumulate) return;
    } else {
        for (int i = threadIdx.x; i < n; i += kThreads) {
            const u32x2 e = a.sorted[first + i];
            key[i] = e[0] << 16 | static_cast<uint32_t>(i);
            tok[i] = e[1];
        }
    }
    if (threadIdx.x < 4) key[n + threadIdx.x] = 0xFFFFFFFFu;
    __syncthreads();
    const int groups = kThreads / a.lanes;
    const int group_rows = (rows + groups - 1) / groups;
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const uint32_t mine = key[i];
        uint32_t rank = 0;
        for (int k = 0; k < n; k += 4) {
            const u32x4 o = *reinterpret_cast<const u32x4*>(&key[k]);
            rank += (o[0] < mine) + (o[1] < mine) + (o[2] < mine) + (o[3] < mine);
        }
        const uint32_t r = mine >> 16;
        row_of[rank] = static_cast<uint16_t>(r);
        by_row[rank] = kDirect ? mine & 0xFFFFu : tok[i];
        atomicOr(&seen[r / 32], 1u << r % 32);
        atomicMax(&group_end[r / group_rows], rank + 1);
    }
    __syncthreads();

    const int lane = threadIdx.x & (a.lanes - 1), g = threadIdx.x / a.lanes;
    const int64_t c = (static_cast<int64_t>(blockIdx.y) * a.lanes + lane) * kVecCols;
    if (item >= 0 && blockIdx.y == 0)
        for (int r = threadIdx.x; r < rows; r += kThreads)
            a.present[static_cast<int64_t>(item) * rows + r] = seen[r / 32] >> r % 32 & 1u;
    if (c >= a.cols) return;
    const int64_t row0 = static_cast<int64_t>(bucket) << a.bits;
    if (item < 0 && !a.accumulate) {
        const float zero[8] = {};
        for (int r = g * group_rows; r < (g + 1) * group_rows && r < rows && row0 + r < a.ids.rows; ++r)
            if (!(seen[r / 32] >> r % 32 & 1u)) finish_row(a, row0 + r, c, zero, false);
    }
    int at = 0;
    for (int k = 0; k < g; ++k) at = max(at, static_cast<int>(group_end[k]));
    const int end = max(at, static_cast<int>(group_end[g]));
    if (at >= end) return;
    const int64_t wide = (a.cols + kVecCols - 1) / kVecCols * kVecCols;
    float acc[8] = {};
    uint32_t cur = row_of[at];
    auto flush = [&]() {
        if (item >= 0) {
            float* p = a.partial + (static_cast<int64_t>(item) * rows + cur) * wide + c;
            *reinterpret_cast<u32x4*>(p) = (u32x4){__float_as_uint(acc[0]), __float_as_uint(acc[1]),
                                                   __float_as_uint(acc[2]), __float_as_uint(acc[3])};
            *reinterpret_cast<u32x4*>(p + 4) = (u32x4){__float_as_uint(acc[4]), __float_as_uint(acc[5]),
                                                       __float_as_uint(acc[6]), __float_as_uint(acc[7])};
        } else {
            finish_row(a, row0 + cur, c, acc, a.accumulate != 0);
        }
    };
    for (; at < end; at += kAhead) {
        Raw<kS> raw[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int i = at + u < end ? at + u : end - 1;
            raw[u] = load8<kS>(a.src + by_row[i] * a.src_stride, c, a.cols);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (at + u >= end) break;
            const uint32_t r = row_of[at + u];
            float x[8];
            widen8<kS>(raw[u], x);
            if (r != cur) {
                flush();
                cur = r;
#pragma unroll
                for (int k = 0; k < 8; ++k) acc[k] = 0.0f;
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) acc[k] += x[k];
        }
    }
    flush();
}

// Rows of the split buckets: their chunks' sums in chunk order.  A block takes
// kThreads / lanes rows; blockIdx.x goes over (split bucket, rows).
__global__ __launch_bounds__(kThreads) void join_kernel(GradArgs a) {
    const int rows = 1 << a.bits;
    const int groups = kThreads / a.lanes;
    const int per = (rows + groups - 1) / groups;  // blocks of a bucket
    const int m = blockIdx.x / per;
    if (m >= a.heads[1]) return;
    const Split s = a.splits[m];
    const int r = (blockIdx.x - m * per) * groups + threadIdx.x / a.lanes;
    const int64_t row = (static_cast<int64_t>(s.bucket) << a.bits) + r;
    const int64_t c = (static_cast<int64_t>(blockIdx.y) * a.lanes + (threadIdx.x & (a.lanes - 1))) * kVecCols;
    if (r >= rows || row >= a.ids.rows || c >= a.cols) return;
    const int64_t wide = (a.cols + kVecCols - 1) / kVecCols * kVecCols;
    float acc[8] = {};
    bool any = false;
    for (int k = 0; k < s.count; ++k) {
        const int64_t at = static_cast<int64_t>(s.item + k) * rows + r;
        if (!a.present[at]) continue;
        any = true;
        const float* p = a.partial + at * wide + c;
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] += p[i];
    }
    if (any || !a.accumulate) finish_row(a, row, c, acc, a.accumulate != 0);
}

// ---- host --------------------------------------------------------------------

constexpr int64_t kMaxRows = int64_t{kMaxBuckets} << kMaxBucketBits;
constexpr int64_t kMaxTokens = INT32_MAX;
constexpr int64_t kMaxCols = int64_t{1} << 24;

// Lanes of a row: the power of two up to kThreads with the fewest idle lanes
// over all column blocks, the larger one of equals.
int lanes_for(int64_t cols) {
    const int64_t need = (cols + kVecCols - 1) / kVecCols;
    int lanes = 1;
    while (lanes < kThreads && lanes < need) lanes *= 2;
    if (need > lanes) {
        int64_t best = (need + lanes - 1) / lanes * lanes;
        for (int l = lanes / 2; l >= 64; l /= 2) {
            const int64_t all = (need + l - 1) / l * l;
            if (all < best) {
                best = all;
                lanes = l;
            }
        }
    }
    return lanes;
}

int col_blocks(int64_t cols, int lanes) {
    return static_cast<int>((cols + int64_t{kVecCols} * lanes - 1) / (int64_t{kVecCols} * lanes));
}

// Shapes of one gradient call: buckets, chunks and the workspace's parts.
struct GradPlan {
    bool direct;
    int bits, buckets, place_blocks, place_tokens, max_items, max_splits;
    size_t counts, starts, heads, items, splits, sorted, present, partial, bytes;
};

GradPlan plan_grad(int64_t tokens, int64_t rows, int64_t cols) {
    GradPlan p{};
    p.bits = kMinBucketBits;
    while ((rows + (int64_t{1} << p.bits) - 1) >> p.bits > kMaxBuckets) ++p.bits;
    p.buckets = static_cast<int>((rows + (int64_t{1} << p.bits) - 1) >> p.bits);
    p.direct = tokens <= kDirectTokens;
    if (p.direct) return p;
    int64_t per = (tokens + kMaxPlaceBlocks - 1) / kMaxPlaceBlocks;
    per = (per + kPlaceThreads - 1) / kPlaceThreads * kPlaceThreads;
    p.place_tokens = static_cast<int>(per);
    p.place_blocks = static_cast<int>((tokens + per - 1) / per);
    // a bucket of n > kChunk tokens has at most n / kChunk + 1 < 2 n / kChunk chunks
    p.max_splits = static_cast<int>(tokens / (kChunk + 1) < p.buckets ? tokens / (kChunk + 1) : p.buckets);
    p.max_items = static_cast<int>(tokens / kChunk) + p.max_splits;
    const int64_t wide = (cols + kVecCols - 1) / kVecCols * kVecCols;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at = (at + bytes + 255) / 256 * 256;
        return here;
    };
    p.counts = take(sizeof(uint32_t) * p.place_blocks * p.buckets);
    p.starts = take(sizeof(uint32_t) * (p.buckets + 1));
    p.heads = take(2 * sizeof(int32_t));
    p.items = take(sizeof(Item) * p.max_items);
    p.splits = take(sizeof(Split) * p.max_splits);
    p.sorted = take(sizeof(u32x2) * tokens);
    p.present = take((size_t{1} << p.bits) * p.max_items);
    p.partial = take((sizeof(float) << p.bits) * p.max_items * static_cast<size_t>(wide));
    p.bytes = at;
    return p;
}

int check_matrix(const char* name, const char* what, const gockpt_matrix* m) {
    if (m == nullptr) return ops_fail(GOCKPT_EINVAL, "%s: null %s", name, what);
    if (!dtype_ok(m->dtype)) return ops_fail(GOCKPT_EINVAL, "%s: %s dtype %d", name, what, m->dtype);
    if (m->rows < 0 || m->cols < 0 || m->rows > kMaxTokens || m->cols > kMaxCols)
        return ops_fail(GOCKPT_EINVAL, "%s: %s of %lld x %lld", name, what, static_cast<long long>(m->rows),
                        static_cast<long long>(m->cols));
    if (m->rows > 1 && (m->stride < m->cols || m->stride > int64_t{1} << 40))
        return ops_fail(GOCKPT_EINVAL, "%s: %s stride %lld for rows of %lld", name, what,
                        static_cast<long long>(m->stride), static_cast<long long>(m->cols));
    if (m->rows > 0 && m->cols > 0 && (m->data == nullptr || !elem_aligned(m->data, m->dtype)))
        return ops_fail(GOCKPT_EINVAL, "%s: %s is null or not aligned to its element", name, what);
    return GOCKPT_OK;
}

// The tokens against a table of `rows` rows and a matrix of one row a token.
int check_ids(const char* name, const gockpt_token_ids* t, int64_t rows, int64_t matrix_rows, Ids* ids) {
    if (t == nullptr) return ops_fail(GOCKPT_EINVAL, "%s: null tokens", name);
    if (t->batch < 0 || t->length < 0 || t->batch > kMaxTokens || t->length > kMaxTokens ||
        t->batch * t->length > kMaxTokens)
        return ops_fail(GOCKPT_EINVAL, "%s: %lld x %lld tokens", name, static_cast<long long>(t->batch),
                        static_cast<long long>(t->length));
    if (t->batch > 1 && (t->stride < t->length || t->stride > int64_t{1} << 31))
        return ops_fail(GOCKPT_EINVAL, "%s: ids stride %lld for sequences of %lld", name,
                        static_cast<long long>(t->stride), static_cast<long long>(t->length));
    if (t->bits != 32 && t->bits != 64) return ops_fail(GOCKPT_EINVAL, "%s: ids of %d bits", name, t->bits);
    const int64_t n = t->batch * t->length;
    if (n > 0 && (t->ids == nullptr || reinterpret_cast<uintptr_t>(t->ids) % (t->bits / 8) != 0))
        return ops_fail(GOCKPT_EINVAL, "%s: ids are null or not aligned", name);
    if (n != matrix_rows)
        return ops_fail(GOCKPT_EINVAL, "%s: %lld tokens, %lld rows", name, static_cast<long long>(n),
                        static_cast<long long>(matrix_rows));
    ids->p = t->ids;
    ids->stride = t->batch > 1 ? t->stride : t->length;
    ids->first = t->first_id;
    ids->padding = INT64_MIN;
    ids->tokens = static_cast<uint32_t>(n);
    ids->length = static_cast<uint32_t>(t->length);
    ids->wide = t->bits == 64;
    ids->rows = static_cast<uint32_t>(rows);
    return GOCKPT_OK;
}

template <int kW>
void launch_lookup(const LookupArgs& a, int out_dtype, dim3 grid, hipStream_t s) {
    if (out_dtype == kBF16)
        hipLaunchKernelGGL((lookup_kernel<kW, kBF16>), grid, dim3(kThreads), 0, s, a);
    else if (out_dtype == kFP16)
        hipLaunchKernelGGL((lookup_kernel<kW, kFP16>), grid, dim3(kThreads), 0, s, a);
    else
        hipLaunchKernelGGL((lookup_kernel<kW, kFP32>), grid, dim3(kThreads), 0, s, a);
}

template <bool kDirect>
void launch_rows(const GradArgs& a, int src_dtype, dim3 grid, hipStream_t s) {
    if (src_dtype == kBF16)
        hipLaunchKernelGGL((rows_kernel<kBF16, kDirect>), grid, dim3(kThreads), 0, s, a);
    else if (src_dtype == kFP16)
        hipLaunchKernelGGL((rows_kernel<kFP16, kDirect>), grid, dim3(kThreads), 0, s, a);
    else
        hipLaunchKernelGGL((rows_kernel<kFP32, kDirect>), grid, dim3(kThreads), 0, s, a);
}

}  // namespace

}  // namespace gockpt

using namespace gockpt;

extern "C" {

int gockpt_embedding(const gockpt_matrix* table, const gockpt_token_ids* tokens, float scale,
                     const gockpt_matrix* out, void* stream) {
    const char* name = "gockpt_embedding";
    LookupArgs a{};
    int rc = check_matrix(name, "table", table);
    if (rc == GOCKPT_OK) rc = check_matrix(name, "out", out);
    if (rc == GOCKPT_OK) rc = check_ids(name, tokens, table->rows, out->rows, &a.ids);
    if (rc != GOCKPT_OK) return rc;
    if (table->cols != out->cols)
        return ops_fail(GOCKPT_EINVAL, "%s: table of %lld columns, out of %lld", name,
                        static_cast<long long>(table->cols), static_cast<long long>(out->cols));
    if (a.ids.tokens == 0 || out->cols == 0) return GOCKPT_OK;
    a.table = static_cast<const uint8_t*>(table->data);
    a.out = static_cast<uint8_t*>(const_cast<void*>(out->data));
    a.cols = table->cols;
    a.table_stride = table->stride * dtype_bytes(table->dtype);
    a.out_stride = out->stride * dtype_bytes(out->dtype);
    a.scale = scale;
    a.lanes = lanes_for(a.cols);
    const uint32_t per = kThreads / a.lanes * kLookupRows;
    const dim3 grid((a.ids.tokens + per - 1) / per, col_blocks(a.cols, a.lanes));
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (table->dtype == kBF16)
        launch_lookup<kBF16>(a, out->dtype, grid, s);
    else if (table->dtype == kFP16)
        launch_lookup<kFP16>(a, out->dtype, grid, s);
    else
        launch_lookup<kFP32>(a, out->dtype, grid, s);
    return ops_launched(name);
}

int gockpt_embedding_grad_bytes(int64_t tokens, int64_t rows, int64_t cols, size_t* bytes) {
    const char* name = "gockpt_embedding_grad_bytes";
    if (bytes == nullptr) return ops_fail(GOCKPT_EINVAL, "%s: null argument", name);
    *bytes = 0;
    if (tokens < 0 || tokens > kMaxTokens || rows < 0 || rows > kMaxRows || cols < 0 || cols > kMaxCols)
        return ops_fail(GOCKPT_EINVAL, "%s: %lld tokens, table of %lld x %lld", name, static_cast<long long>(tokens),
                        static_cast<long long>(rows), static_cast<long long>(cols));
    *bytes = plan_grad(tokens, rows, cols).bytes;
    return GOCKPT_OK;
}

int gockpt_embedding_grad(const gockpt_matrix* grad_out, const gockpt_token_ids* tokens, int64_t padding_id,
                          float scale, int accumulate, const gockpt_matrix* grad_table, void* workspace,
                          size_t workspace_bytes, void* stream) {
    const char* name = "gockpt_embedding_grad";
    GradArgs a{};
    int rc = check_matrix(name, "grad_out", grad_out);
    if (rc == GOCKPT_OK) rc = check_matrix(name, "grad_table", grad_table);
    if (rc == GOCKPT_OK && grad_table->rows > kMaxRows)
        rc = ops_fail(GOCKPT_EINVAL, "%s: table of %lld rows", name, static_cast<long long>(grad_table->rows));
    if (rc == GOCKPT_OK) rc = check_ids(name, tokens, grad_table->rows, grad_out->rows, &a.ids);
    if (rc != GOCKPT_OK) return rc;
    if (grad_table->cols != grad_out->cols)
        return ops_fail(GOCKPT_EINVAL, "%s: grad_out of %lld columns, table of %lld", name,
                        static_cast<long long>(grad_out->cols), static_cast<long long>(grad_table->cols));
    if (grad_table->rows == 0 || grad_table->cols == 0) return GOCKPT_OK;
    if (accumulate && a.ids.tokens == 0) return GOCKPT_OK;
    const GradPlan p = plan_grad(a.ids.tokens, grad_table->rows, grad_table->cols);
    if (p.bytes > 0) {
        if (workspace == nullptr || reinterpret_cast<uintptr_t>(workspace) % 256 != 0)
            return ops_fail(GOCKPT_EINVAL, "%s: the workspace must be 256-byte aligned", name);
        if (workspace_bytes < p.bytes)
            return ops_fail(GOCKPT_ENOMEM, "%s: workspace of %zu bytes, %zu needed", name, workspace_bytes, p.bytes);
    }
    a.ids.padding = padding_id;
    a.src = static_cast<const uint8_t*>(grad_out->data);
    a.dst = static_cast<uint8_t*>(const_cast<void*>(grad_table->data));
    a.cols = grad_table->cols;
    a.src_stride = grad_out->stride * dtype_bytes(grad_out->dtype);
    a.dst_stride = grad_table->stride * dtype_bytes(grad_table->dtype);
    a.scale = scale;
    a.dst_dtype = grad_table->dtype;
    a.accumulate = accumulate != 0;
    a.lanes = lanes_for(a.cols);
    a.bits = p.bits;
    a.buckets = p.buckets;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const unsigned cols = static_cast<unsigned>(col_blocks(a.cols, a.lanes));
    if (p.direct) {
        launch_rows<true>(a, grad_out->dtype, dim3(p.buckets, cols), s);
        return ops_launched(name);
    }
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    a.place_blocks = p.place_blocks;
    a.place_tokens = p.place_tokens;
    a.max_items = p.max_items;
    a.max_splits = p.max_splits;
    a.counts = reinterpret_cast<uint32_t*>(ws + p.counts);
    a.starts = reinterpret_cast<uint32_t*>(ws + p.starts);
    a.heads = reinterpret_cast<int32_t*>(ws + p.heads);
    a.items = reinterpret_cast<Item*>(ws + p.items);
    a.splits = reinterpret_cast<Split*>(ws + p.splits);
    a.sorted = reinterpret_cast<u32x2*>(ws + p.sorted);
    a.present = ws + p.present;
    a.partial = reinterpret_cast<float*>(ws + p.partial);
    hipLaunchKernelGGL(count_kernel, dim3(p.place_blocks), dim3(kPlaceThreads), 0, s, a);
    hipLaunchKernelGGL(place_kernel, dim3(p.place_blocks), dim3(kPlaceThreads), 0, s, a);
    launch_rows<false>(a, grad_out->dtype, dim3(p.max_items + p.buckets, cols), s);
    if (p.max_splits > 0) {
        const int groups = kThreads / a.lanes, rows = 1 << a.bits;
        const unsigned per = static_cast<unsigned>((rows + groups - 1) / groups);
        hipLaunchKernelGGL(join_kernel, dim3(p.max_splits * per, cols), dim3(kThreads), 0, s, a);
    }
    return ops_launched(name);
}

}  // extern "C"
