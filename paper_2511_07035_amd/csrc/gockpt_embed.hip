// gockpt_embed.hip -- embedding lookup with scaling, and its gradient.
//
//   lookup_kernel  out[t] = round(scale * table[id[t]]), zeros for masked ids.
//
//   The gradient of row v is scale * (sum of grad_out over the tokens with id
//   v): a sum over tokens sorted by row, in token order within a row.
//   direct_kernel  few tokens, one launch: every block looks through all ids
//                  for those of its 64 rows.
//   bucket_kernel  sorts up to 8192 tokens in one launch, and
//   count_kernel, place_kernel  any number, in one radix pass or two.
//   sum_kernel     sums equal chunks of the sorted tokens row by row in
//                  registers, however many tokens a row has, and writes the rows;
//   join_kernel    adds up the rows that lie in several chunks.
//   No atomics on sums, and chunks by place alone: the same bits every time.
//
//   Memory bounds it: grad_out read once, every row of the table written.
//   131072 tokens x 4096 fp16 into 32000 rows, a tenth masked (0.97 GB + 0.26
//   GB): 271 us, of which the sort 32 (half of the table is cleared meanwhile),
//   the sums 223 at 5.4 TB/s, the join 16.  16384 x 2048 bf16 into 50304 rows
//   (67 + 206 MB): 62 us; accumulated, with no zeros to write, 58.  A copy moves
//   the bytes of the first two in 260 and 58.
#include <limits.h>

#include "gockpt_ops_internal.h"

#pragma clang fp contract(off)

namespace gockpt {

namespace {

constexpr int kThreads = 256;
struct Ids {
    const void* p;
    int64_t stride, first;
    int64_t padding;   // id that adds nothing to a gradient
    uint32_t tokens, length;
    int32_t wide;      // 64-bit ids
    uint32_t rows;     // of the table, at most INT32_MAX
    uint32_t magic;    // floor(2^32 / length), or 2^32 - 1
};

// Row of token t (t < tokens), or -1 where it is masked.
__device__ __forceinline__ int32_t token_row(const Ids& ids, uint32_t t, bool grad) {
    int64_t at = t;
    if (ids.stride != ids.length) {
        // the high word falls short of t / length by at most 1: t < 2^31
        const uint32_t b = __umulhi(t, ids.magic), l = t - b * ids.length;
        at = b * ids.stride + l;
        if (l >= ids.length) at += ids.stride - ids.length;
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
    int32_t lanes;       // of a row, a power of two
    uint32_t col_blocks;
};

// kV adjacent columns c to c + kV - 1 of a row, zeros from `cols` on.
template <int kT, int kV>
struct Piece {
    static constexpr int kWords = kV * (kT == kFP32 ? 4 : 2) / 4;
    uint32_t w[kWords];

    template <bool kNT = false>
    __device__ __forceinline__ void load(const uint8_t* p, int64_t c, int64_t cols) {
        p += c * (kT == kFP32 ? 4 : 2);
        if (c + kV <= cols) {
            if constexpr (kWords == 2) {
                const u32x2_any* at = reinterpret_cast<const u32x2_any*>(p);
                const u32x2 x = kNT ? __builtin_nontemporal_load(at) : *at;
                w[0] = x[0], w[1] = x[1];
            } else {
#pragma unroll
                for (int i = 0; i < kWords; i += 4) {
                    const u32x4_any* at = reinterpret_cast<const u32x4_any*>(p + 4 * i);
                    const u32x4 x = kNT ? __builtin_nontemporal_load(at) : *at;
                    w[i] = x[0], w[i + 1] = x[1], w[i + 2] = x[2], w[i + 3] = x[3];
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < kWords; ++i) w[i] = 0u;
#pragma unroll
            for (int i = 0; i < kV - 1; ++i) {
                if (c + i >= cols) break;
                if constexpr (kT == kFP32)
                    w[i] = reinterpret_cast<const uint32_t*>(p)[i];
                else
                    w[i / 2] |= static_cast<uint32_t>(reinterpret_cast<const uint16_t*>(p)[i]) << (16 * (i % 2));
            }
        }
    }
    __device__ __forceinline__ float operator[](int i) const {
        if constexpr (kT == kFP32)
            return __uint_as_float(w[i]);
        else
            return elem_to_f32<kT>(w[i / 2] >> (16 * (i % 2)) & 0xFFFFu);
    }
};

// kV columns of a row at p from column c on.
template <int kT, int kV, bool kNT>
__device__ __forceinline__ void store_cols(uint8_t* p, int64_t c, int64_t cols, const float* x) {
    constexpr int kB = kT == kFP32 ? 4 : 2;
    constexpr int kWords = kV * kB / 4;
    p += c * kB;
    if (c + kV <= cols) {
        uint32_t w[kWords];
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            if constexpr (kT == kFP32)
                w[i] = __float_as_uint(x[i]);
            else
                w[i] = pack2<kT>(x[2 * i], x[2 * i + 1]);
        }
        if constexpr (kWords == 2) {
            *reinterpret_cast<u32x2_any*>(p) = (u32x2){w[0], w[1]};
        } else {
#pragma unroll
            for (int i = 0; i < kWords; i += 4) {
                const u32x4 v = {w[i], w[i + 1], w[i + 2], w[i + 3]};
                if constexpr (kNT)
                    __builtin_nontemporal_store(v, reinterpret_cast<u32x4_any*>(p + 4 * i));
                else
                    *reinterpret_cast<u32x4_any*>(p + 4 * i) = v;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < kV - 1; ++i)
            if (c + i < cols) store_elem<kT>(p + kB * i, x[i]);
    }
}

// A lane takes 16 bytes of output columns, so that a wavefront's stores are one
// contiguous KiB (fp32 output at 8 columns a lane, two stores 32 bytes apart,
// ran at half the rate).  A piece is kThreads / lanes rows in one column block;
// a block takes kPieces of them, all columns of a row before the next row, and
// has all their loads in flight before its first store.
//
// Bound by the writes, and by the reads of rows that the caches do not hold:
// 65536 x 5120 fp32 from a bf16 table whose rows lie in HBM 345 us, with them
// in the last-level cache 250 (1.34 GB written: 195 us at the rate of a fill,
// 312 at a copy's over all 1.48 GB); 131072 x 4096 bf16 287, 16384 x 2048 bf16
// 19.  us with 2, 3, 4 and 8 pieces: 396, 338, 345, 355; 310, 302, 287, 325;
// 18.8, 19.0, 19.3, 21.9: with 4 each is within 3% of its best, with the others
// one is 5% off or more.  Slower: the same column block of several rows in a
// block (357, 310); a row's column blocks on one XCD each, so that its L2 holds
// parts of more rows; contiguous tokens on each XCD; loads past the caches
// (389); stores written through the L2.
constexpr int kPieces = 4;

template <int kW, int kO, bool kNT>
__global__ __launch_bounds__(kThreads) void lookup_kernel(LookupArgs a) {
    constexpr int kV = kO == kFP32 ? 4 : 8;
    const uint32_t lane = threadIdx.x & (a.lanes - 1);
    const uint32_t per = kThreads / a.lanes;
    uint32_t group = blockIdx.x * kPieces / a.col_blocks, col = blockIdx.x * kPieces - group * a.col_blocks;
    int32_t row[kPieces];
    uint32_t t[kPieces];
    int64_t c[kPieces];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
        t[i] = group * per + threadIdx.x / a.lanes;
        c[i] = (static_cast<int64_t>(col) * a.lanes + lane) * kV;
        row[i] = t[i] < a.ids.tokens ? token_row(a.ids, t[i], false) : -1;
        if (++col == a.col_blocks) {
            col = 0;
            ++group;
        }
    }
    Piece<kW, kV> x[kPieces] = {};
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
        if (row[i] >= 0) x[i].load(a.table + row[i] * a.table_stride, c[i], a.cols);
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
        if (t[i] >= a.ids.tokens) continue;
        float y[kV];
        // a masked token's zeros stay +0 whatever the scale
#pragma unroll
        for (int k = 0; k < kV; ++k) y[k] = row[i] >= 0 ? x[i][k] * a.scale : 0.0f;
        store_cols<kO, kV, kNT>(a.out + t[i] * a.out_stride, c[i], a.cols, y);
    }
}

// ---- gradient ----------------------------------------------------------------

constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kMaxDigits = 2048;
constexpr int kMaxSortBlocks = 64;
// Up to this many tokens take direct_kernel.  Its blocks read a row's tokens one
// after the other, so a row that has most of them bounds it: us direct and
// sorted, bf16, 50304 x 2048, ids by text's law: 16 tokens 44 and 49, 128 50.5
// and 57.5, 256 60.6 and 57.7, 1024 124 and 58.5; fp32, 320 x 64: 128 8.0 and
// 19.5 with ids of one chance, 24 and 14 all of one id.
constexpr int kDirectTokens = 128;
// Up to this many take bucket_kernel, one launch instead of four: 2048 tokens
// into 50304 x 2048 47.7 and 54.8, 8192 55.3 and 58.1, 16384 76 and 71.
constexpr int kBucketTokens = 8192;
constexpr int kBucketDigits = 512;
// Bytes of the table that are cleared beside the sort: 96 MiB beside
// bucket_kernel, 32 beside each of the four radix launches.  The rows that have
// a token are written again, and the writes slow the sort, so more is not
// better: us with 24, 32 and 48 MiB a launch, 16384 tokens into 206 MB 65.8,
// 65.3, 68.8, 131072 into 262 MB 273, 272, 278; with 64, 96 and 128, 8192 tokens
// 54.8, 50.9, 52.1.  A table above kCachedOutBytes is cleared past the caches
// (with plain stores 72.8, 273 and 54.7).
constexpr int64_t kClearBucketBytes = int64_t{96} << 20;
constexpr int64_t kClearRadixBytes = int64_t{32} << 20;
// Blocks that do it (64, 256 and 512: 68.2, 68.9, 66.7 us for the 16384).
constexpr int kClearBlocks = 128;

// A token and its row.
struct alignas(8) Pair {
    uint32_t row, token;
};

struct GradArgs {
    Ids ids;
    const uint8_t* src;
    uint8_t* dst;
    int64_t cols, src_stride, dst_stride;  // strides in bytes
    float scale;
    int32_t dst_dtype, accumulate;
    int32_t lanes;                         // of a row, a power of two
    uint32_t col_blocks;
    // blocks of a launch that sort, and tokens of each; the others clear a part
    // of the table
    int32_t sort_blocks, sort_tokens;
    int32_t digits;                        // of the running radix pass
    uint32_t shift;
    // Rows from clear_from on are cleared in `parts` parts by the launches that
    // sort (whose blocks alone leave most of the device idle), before it is
    // known which have a token; the others, where none has, by sum_kernel's
    // blocks from sum_blocks on.
    int64_t clear_from;
    bool clear_nt;
    int32_t part, parts;
    uint32_t sum_blocks;
    int32_t chunk;                         // sorted tokens that one group of lanes sums
    // workspace
    uint32_t* heads;                       // tokens that count
    uint32_t* counts;                      // [sort_blocks][digits]
    Pair* first;                           // after the first of two passes
    Pair* sorted;
    float* partial;                        // [2 * chunks][wide]
    int64_t wide;                          // cols rounded up to 8
};

// Zeros `bytes` at p (2-byte aligned, a multiple of 2) with n threads, this one
// number i; past the caches with nt.
__device__ __forceinline__ void clear_span(uint8_t* p, int64_t bytes, uint32_t i, uint32_t n, bool nt) {
    const u32x4 zero = {0u, 0u, 0u, 0u};
    if (nt) {
        for (int64_t at = i * 16; at + 16 <= bytes; at += n * 16)
            __builtin_nontemporal_store(zero, reinterpret_cast<u32x4_any*>(p + at));
    } else {
        for (int64_t at = i * 16; at + 16 <= bytes; at += n * 16) *reinterpret_cast<u32x4_any*>(p + at) = zero;
    }
    const int64_t tail = bytes / 16 * 16 + i * 2;
    if (tail < bytes) *reinterpret_cast<uint16_t*>(p + tail) = 0;
}

// This block's share of the launch's part of the rows from a.clear_from on.
__device__ __forceinline__ void clear_table(const GradArgs& a) {
    const int64_t rows = a.ids.rows - a.clear_from, blocks = int64_t{gridDim.x} - a.sort_blocks;
    const int64_t i = int64_t{blockIdx.x} - a.sort_blocks;
    const int64_t lo = a.clear_from + rows * a.part / a.parts, hi = a.clear_from + rows * (a.part + 1) / a.parts;
    const int64_t r0 = lo + (hi - lo) * i / blocks, r1 = lo + (hi - lo) * (i + 1) / blocks;
    const int64_t bytes = a.cols * (a.dst_dtype == kFP32 ? 4 : 2);
    if (a.dst_stride == bytes) {
        clear_span(a.dst + r0 * bytes, (r1 - r0) * bytes, threadIdx.x, kSortThreads, a.clear_nt);
    } else {
        for (int64_t r = r0 + threadIdx.x / 64; r < r1; r += kSortWaves)
            clear_span(a.dst + r * a.dst_stride, bytes, threadIdx.x & 63, 64, a.clear_nt);
    }
}

// Turns the counts in total[0, digits) into each digit's first place (counts of
// all smaller digits); returns their sum.  Whole block; ends with a barrier.
template <int kDigits>
__device__ __forceinline__ uint32_t digit_starts(uint32_t (&total)[kDigits], int digits) {
    __shared__ uint32_t wave_sum[kSortWaves];
    constexpr int kPer = kDigits > kSortThreads ? kDigits / kSortThreads : 1;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, d0 = threadIdx.x * kPer;
    uint32_t x[kPer], s = 0;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        x[k] = d0 + k < digits ? total[d0 + k] : 0u;
        s += x[k];
    }
    uint32_t at = s;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t y = __shfl_up(at, o, 64);
        if (lane >= o) at += y;
    }
    if (lane == 63) wave_sum[w] = at;
    __syncthreads();
    at -= s;
    uint32_t all = 0;
#pragma unroll
    for (int k = 0; k < kSortWaves; ++k) {
        if (k < w) at += wave_sum[k];
        all += wave_sum[k];
    }
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        if (d0 + k < digits) total[d0 + k] = at;
        at += x[k];
    }
    __syncthreads();
    return all;
}

// Tokens of each digit in each wavefront's 64: a byte each, a digit's 16 bytes
// one LDS read.
template <int kDigits>
struct WaveCounts {
    uint8_t n[kDigits][kSortWaves];

    __device__ __forceinline__ void clear(int digits) {
        const u32x4 zero = {0u, 0u, 0u, 0u};
        for (int d = threadIdx.x; d < digits; d += kSortThreads) *reinterpret_cast<u32x4*>(n[d]) = zero;
    }
    // The sum over the wavefronts before w.
    __device__ __forceinline__ uint32_t before(uint32_t d, int w) const {
        const u32x4 x = *reinterpret_cast<const u32x4*>(n[d]);
        uint32_t s = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int bytes = w - 4 * j;
            const uint32_t mask = bytes >= 4 ? ~0u : bytes <= 0 ? 0u : (1u << 8 * bytes) - 1u;
            s = __builtin_amdgcn_sad_u8(x[j] & mask, 0u, s);
        }
        return s;
    }
};
static_assert(kSortWaves == 16, "16 bytes a digit");

// One token of each thread to its digit's next place, in thread order within a
// digit.  in_wave: zero before, and again after the next barrier.  Whole block.
template <int kDigits, class Out>
__device__ __forceinline__ void place_round(uint32_t (&next)[kDigits], WaveCounts<kDigits>& in_wave, int digits,
                                            bool there, uint32_t d, Out&& out) {
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint64_t same = __ballot(there);  // the lanes of this wavefront with the same digit
    for (int b = 0; (digits - 1) >> b; ++b) {
        const bool bit = d >> b & 1u;
        const uint64_t m = __ballot(bit);
        same &= bit ? m : ~m;
    }
    const int rank = __popcll(same & ((uint64_t{1} << lane) - 1));
    const bool leads = there && rank == 0;
    if (leads) in_wave.n[d][w] = static_cast<uint8_t>(__popcll(same));
    __syncthreads();
    if (there) out(next[d] + in_wave.before(d, w) + rank);
    __syncthreads();
    if (leads) {
        atomicAdd(&next[d], static_cast<uint32_t>(__popcll(same)));
        in_wave.n[d][w] = 0;
    }
}

// Sort of at most kBucketTokens tokens in one launch: a block takes the rows of
// one bucket of 1 << bits, at most kBucketDigits.  It looks through all ids,
// counts the tokens of smaller rows, which is where its own begin, lists its own
// in token order and sorts them by row in one counting pass.
constexpr uint32_t kIdsAhead = 8;

__global__ __launch_bounds__(kSortThreads, 8) void bucket_kernel(GradArgs a, int bits) {
    constexpr int kDigits = kBucketDigits;
    __shared__ uint32_t list[kBucketTokens];  // row within the bucket << 16 | token
    __shared__ uint32_t next[kDigits];
    __shared__ alignas(16) WaveCounts<kDigits> in_wave;
    __shared__ uint32_t found[kSortWaves], below[kSortWaves], valid[kSortWaves];
    if (static_cast<int>(blockIdx.x) >= a.sort_blocks) {
        clear_table(a);
        return;
    }
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int digits = 1 << bits, bucket = blockIdx.x;
    // a wavefront's tokens follow one another
    const uint32_t n = a.ids.tokens, rounds = (n + kSortThreads - 1) / kSortThreads, t0 = w * rounds * 64 + lane;
    // f(row, token) round by round, the ids of kIdsAhead rounds loaded together
    auto each_round = [&](auto&& f) {
        for (uint32_t r0 = 0; r0 < rounds; r0 += kIdsAhead) {
            int32_t row[kIdsAhead];
#pragma unroll
            for (uint32_t k = 0; k < kIdsAhead; ++k) {
                const uint32_t t = t0 + (r0 + k) * 64;
                row[k] = r0 + k < rounds && t < n ? token_row(a.ids, t, true) : -1;
            }
#pragma unroll
            for (uint32_t k = 0; k < kIdsAhead; ++k) f(row[k], t0 + (r0 + k) * 64);
        }
    };
    uint32_t mine = 0, less = 0, all = 0;
    each_round([&](int32_t row, uint32_t) {
        mine += __popcll(__ballot(row >> bits == bucket));
        less += __popcll(__ballot(row >= 0 && row >> bits < bucket));
        all += __popcll(__ballot(row >= 0));
    });
    if (lane == 0) found[w] = mine, below[w] = less, valid[w] = all;
    for (int d = threadIdx.x; d < digits; d += kSortThreads) next[d] = 0u;
    in_wave.clear(digits);
    __syncthreads();
    uint32_t at = 0, count = 0, base = 0, total = 0;
#pragma unroll
    for (int k = 0; k < kSortWaves; ++k) {
        if (k < w) at += found[k];
        count += found[k];
        base += below[k];
        total += valid[k];
    }
    if (bucket == 0 && threadIdx.x == 0) a.heads[0] = total;
    if (count == 0) return;
    each_round([&](int32_t row, uint32_t t) {  // the ids again, from the L2
        const bool in = row >> bits == bucket;
        const uint64_t m = __ballot(in);
        if (in) {
            const uint32_t d = static_cast<uint32_t>(row) & (digits - 1);
            list[at + __popcll(m & ((uint64_t{1} << lane) - 1))] = d << 16 | t;
            atomicAdd(&next[d], 1u);
        }
        at += __popcll(m);
    });
    __syncthreads();
    digit_starts(next, digits);
    Pair* out = a.sorted + base;
    const uint32_t row0 = static_cast<uint32_t>(bucket) << bits;
    for (uint32_t i = 0; i < count; i += kSortThreads) {
        const bool there = i + threadIdx.x < count;
        const uint32_t e = there ? list[i + threadIdx.x] : 0u;
        place_round(next, in_wave, digits, there, e >> 16,
                    [&](uint32_t to) { out[to] = {row0 + (e >> 16), e & 0xFFFFu}; });
    }
}

// Radix sort, stable, in one pass over the row's bits or two (low ones first).
// kFirst: the pass reads the ids; masked tokens drop out.
template <bool kFirst>
__device__ __forceinline__ bool sort_input(const GradArgs& a, const Pair* in, uint32_t i, uint32_t n, Pair& p) {
    if (i >= n) return false;
    if constexpr (kFirst) {
        const int32_t row = token_row(a.ids, i, true);
        p = {static_cast<uint32_t>(row), i};
        return row >= 0;
    } else {
        p = in[i];
        return true;
    }
}

template <bool kFirst>
__global__ __launch_bounds__(kSortThreads) void count_kernel(GradArgs a) {
    __shared__ uint32_t n[kMaxDigits];
    if (static_cast<int>(blockIdx.x) >= a.sort_blocks) {
        clear_table(a);
        return;
    }
    for (int d = threadIdx.x; d < a.digits; d += kSortThreads) n[d] = 0u;
    __syncthreads();
    const uint32_t all = kFirst ? a.ids.tokens : a.heads[0];
    const uint32_t t0 = blockIdx.x * static_cast<uint32_t>(a.sort_tokens);
    for (int i = threadIdx.x; i < a.sort_tokens; i += kSortThreads) {
        Pair p;
        if (sort_input<kFirst>(a, a.first, t0 + i, all, p)) atomicAdd(&n[p.row >> a.shift & (a.digits - 1)], 1u);
    }
    __syncthreads();
    for (int d = threadIdx.x; d < a.digits; d += kSortThreads) a.counts[blockIdx.x * a.digits + d] = n[d];
}

// Writes the block's tokens to their places.
template <bool kFirst>
__global__ __launch_bounds__(kSortThreads) void place_kernel(GradArgs a, Pair* out) {
    __shared__ uint32_t next[kMaxDigits];    // tokens of each digit, then the next place of each for this block
    __shared__ uint32_t before[kMaxDigits];  // tokens in earlier blocks
    __shared__ alignas(16) WaveCounts<kMaxDigits> in_wave;
    if (static_cast<int>(blockIdx.x) >= a.sort_blocks) {
        clear_table(a);
        return;
    }
    const int digits = a.digits;
    const uint32_t n = kFirst ? a.ids.tokens : a.heads[0];
    const uint32_t t0 = blockIdx.x * static_cast<uint32_t>(a.sort_tokens) + threadIdx.x;
    Pair p = {0u, 0u};
    bool there = sort_input<kFirst>(a, a.first, t0, n, p);  // on its way while the counts are read
    for (int d = threadIdx.x; d < digits; d += kSortThreads) next[d] = before[d] = 0u;
    in_wave.clear(digits);
    __syncthreads();
    const int groups = digits < kSortThreads ? kSortThreads / digits : 1;
    for (int d = threadIdx.x & (digits - 1); d < digits; d += kSortThreads) {
        uint32_t sum = 0, earlier = 0;
#pragma unroll 8
        for (int b = digits < kSortThreads ? threadIdx.x / digits : 0; b < a.sort_blocks; b += groups) {
            const uint32_t n = a.counts[b * digits + d];
            sum += n;
            if (b < static_cast<int>(blockIdx.x)) earlier += n;
        }
        atomicAdd(&next[d], sum);
        atomicAdd(&before[d], earlier);
    }
    __syncthreads();
    const uint32_t all = digit_starts(next, digits);
    for (int d = threadIdx.x; d < digits; d += kSortThreads) next[d] += before[d];
    if (kFirst && blockIdx.x == 0 && threadIdx.x == 0) a.heads[0] = all;
    __syncthreads();
    for (int i = kSortThreads;; i += kSortThreads) {
        const Pair now = p;
        const bool is = there;
        if (i < a.sort_tokens) there = sort_input<kFirst>(a, a.first, t0 + i, n, p);
        place_round(next, in_wave, digits, is, now.row >> a.shift & (digits - 1), [&](uint32_t at) { out[at] = now; });
        if (i >= a.sort_tokens) break;
    }
}

// kV columns from c on of a row of the table: scale * acc, or that and what is
// there.
template <int kD, int kV>
__device__ __forceinline__ void finish_as(const GradArgs& a, int64_t row, int64_t c, const float (&acc)[kV],
                                           bool add) {
    uint8_t* p = a.dst + row * a.dst_stride;
    float x[kV];
#pragma unroll
    for (int k = 0; k < kV; ++k) x[k] = acc[k] * a.scale;
    if (add) {
        Piece<kD, kV> old;
        old.load(p, c, a.cols);
#pragma unroll
        for (int k = 0; k < kV; ++k) x[k] = old[k] + x[k];
    }
    store_cols<kD, kV, false>(p, c, a.cols, x);
}

template <int kV>
__device__ __forceinline__ void finish_row(const GradArgs& a, int64_t row, int64_t c, const float (&acc)[kV],
                                           bool add) {
    if (a.dst_dtype == kBF16)
        finish_as<kBF16, kV>(a, row, c, acc, add);
    else if (a.dst_dtype == kFP16)
        finish_as<kFP16, kV>(a, row, c, acc, add);
    else
        finish_as<kFP32, kV>(a, row, c, acc, add);
}

// Tokens whose loads a lane has in flight.  sum_kernel issues the next one as
// each is added; 4, 8 and 16: 131072 x 4096 377, 377, 380 us.
constexpr int kDirectAhead = 8;
constexpr int kAhead = 8;
constexpr int kMaxChunk = 64;   // a pair a lane
constexpr int kMinLanes = 16;   // lanes of a row in sum_kernel and join_kernel

// One bucket of kBucketRows rows, all its tokens: found among all ids, sorted by
// (row, token) in LDS by counting, for each, the smaller keys, then summed row
// by row.  A row is `lanes` lanes wide, and the block's groups of so many lanes
// take equal ranges of rows.
constexpr int kBucketRows = 64;

template <int kS>
__global__ __launch_bounds__(kThreads) void direct_kernel(GradArgs a) {
    constexpr int kV = kS == kFP32 ? 4 : 8;
    __shared__ alignas(16) uint32_t key[kDirectTokens + 4];  // row << 16 | token
    __shared__ uint32_t sorted[kDirectTokens];
    __shared__ uint32_t seen[kBucketRows / 32];
    __shared__ int group_end[kThreads];
    __shared__ uint32_t found;

    const uint32_t bucket = blockIdx.x / a.col_blocks, col = blockIdx.x - bucket * a.col_blocks;
    const int64_t row0 = int64_t{bucket} * kBucketRows;
    if (threadIdx.x < kBucketRows / 32) seen[threadIdx.x] = 0u;
    group_end[threadIdx.x] = 0;
    if (threadIdx.x == 0) found = 0u;
    __syncthreads();
    for (uint32_t t = threadIdx.x; t < a.ids.tokens; t += kThreads) {
        const uint32_t r = static_cast<uint32_t>(token_row(a.ids, t, true) - static_cast<int32_t>(row0));
        if (r < kBucketRows) key[atomicAdd(&found, 1u)] = r << 16 | t;
    }
    __syncthreads();
    const int n = static_cast<int>(found);
    if (n == 0 && a.accumulate) return;
    if (threadIdx.x < 4) key[n + threadIdx.x] = 0xFFFFFFFFu;
    __syncthreads();
    const int groups = kThreads / a.lanes;
    const int group_rows = (kBucketRows + groups - 1) / groups;
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const uint32_t mine = key[i];
        int rank = 0;
        for (int k = 0; k < n; k += 4) {
            const u32x4 o = *reinterpret_cast<const u32x4*>(&key[k]);
            rank += (o[0] < mine) + (o[1] < mine) + (o[2] < mine) + (o[3] < mine);
        }
        sorted[rank] = mine;
        const uint32_t r = mine >> 16;
        atomicOr(&seen[r / 32], 1u << r % 32);
        atomicMax(&group_end[r / group_rows], rank + 1);
    }
    __syncthreads();

    const int lane = threadIdx.x & (a.lanes - 1), g = threadIdx.x / a.lanes;
    const int64_t c0 = static_cast<int64_t>(col) * a.lanes * kV, c = c0 + lane * kV;
    if (!a.accumulate) {  // rows without a token, a wavefront each
        const int64_t wide = a.lanes * kV, size = a.dst_dtype == kFP32 ? 4 : 2;
        const int64_t bytes = (a.cols - c0 < wide ? a.cols - c0 : wide) * size;
        const int64_t here = a.ids.rows - row0 < kBucketRows ? a.ids.rows - row0 : kBucketRows;
        if (n == 0 && bytes == a.dst_stride) {
            clear_span(a.dst + row0 * bytes, here * bytes, threadIdx.x, kThreads, a.clear_nt);
            return;
        }
        for (int r = threadIdx.x / 64; r < here; r += kThreads / 64)
            if (!(seen[r / 32] >> r % 32 & 1u))
                clear_span(a.dst + (row0 + r) * a.dst_stride + c0 * size, bytes, threadIdx.x & 63, 64, a.clear_nt);
    }
    if (c >= a.cols) return;
    int at = 0;
    for (int k = 0; k < g; ++k) at = max(at, group_end[k]);
    const int end = max(at, group_end[g]);
    if (at >= end) return;
    float acc[kV] = {};
    uint32_t cur = sorted[at] >> 16;
    for (; at < end; at += kDirectAhead) {
        Piece<kS, kV> x[kDirectAhead];
#pragma unroll
        for (int u = 0; u < kDirectAhead; ++u) {
            const int i = at + u < end ? at + u : end - 1;
            x[u].load(a.src + (sorted[i] & 0xFFFFu) * a.src_stride, c, a.cols);
        }
#pragma unroll
        for (int u = 0; u < kDirectAhead; ++u) {
            if (at + u >= end) break;
            const uint32_t r = sorted[at + u] >> 16;
            if (r != cur) {
                finish_row<kV>(a, row0 + cur, c, acc, a.accumulate != 0);
                cur = r;
#pragma unroll
                for (int k = 0; k < kV; ++k) acc[k] = 0.0f;
            }
#pragma unroll
            for (int k = 0; k < kV; ++k) acc[k] += x[u][k];
        }
    }
    finish_row<kV>(a, row0 + cur, c, acc, a.accumulate != 0);
}

constexpr int kClearRows = 64;  // of a block that clears absent rows

// Clears those of 64 rows below clear_from that no token has: a lane looks its
// row up among the sorted tokens.
__device__ __forceinline__ void clear_absent(const GradArgs& a, uint32_t block) {
    const int lane = threadIdx.x & 63;
    const int64_t row0 = int64_t{block} * kClearRows;
    const uint32_t row = static_cast<uint32_t>(row0) + lane, n = a.heads[0];
    uint32_t lo = 0, hi = n;  // the first token whose row is not below `row`
    while (lo < hi) {
        const uint32_t mid = lo + (hi - lo) / 2;
        if (a.sorted[mid].row < row)
            lo = mid + 1;
        else
            hi = mid;
    }
    const uint64_t there = __ballot(lo < n && a.sorted[lo].row == row);
    const int64_t bytes = a.cols * (a.dst_dtype == kFP32 ? 4 : 2);
    const int64_t here = a.clear_from - row0 < kClearRows ? a.clear_from - row0 : kClearRows;
    if ((there & (here < 64 ? (uint64_t{1} << here) - 1 : ~uint64_t{0})) == 0 && bytes == a.dst_stride) {
        clear_span(a.dst + row0 * bytes, here * bytes, threadIdx.x, kThreads, a.clear_nt);
        return;
    }
    for (int r = threadIdx.x / 64; r < here; r += kThreads / 64)
        if (!(there >> r & 1u)) clear_span(a.dst + (row0 + r) * a.dst_stride, bytes, lane, 64, a.clear_nt);
}

// Sorted tokens q * chunk to q * chunk + chunk - 1, summed row by row by
// `lanes` lanes, kV columns each.  A row that lies in this chunk alone is
// finished here; of one that began before, the sum goes to partial 2 q, of one
// that begins here and goes on, to 2 q + 1.  Sums that are added to what the table
// holds (kAdd) are a kernel apart, which keeps the plain one's registers at 70, not
// 90: 16384 tokens into 50304 x 2048 62 us, 64.5 as one.  What a row holds is loaded
// when the row ends; loading it when the row begins was no faster (59 us, 58).
template <int kS, bool kWave, bool kAdd>
__global__ __launch_bounds__(kThreads) void sum_kernel(GradArgs a) {
    constexpr int kV = kS == kFP32 ? 4 : 8;
    __shared__ Pair pairs[kWave ? 1 : kThreads / kMinLanes * kMaxChunk];
    if (blockIdx.x >= a.sum_blocks) {
        clear_absent(a, blockIdx.x - a.sum_blocks);
        return;
    }
    const int lane = threadIdx.x & (a.lanes - 1), g = threadIdx.x / a.lanes;
    // a block's groups take the column blocks of a chunk, then the next chunk:
    // groups of one wavefront mostly end rows together
    const uint32_t n = a.heads[0], item = blockIdx.x * (kThreads / a.lanes) + g;
    uint32_t q = item / a.col_blocks;
    if constexpr (kWave) q = __builtin_amdgcn_readfirstlane(q);
    const uint32_t col = item - q * a.col_blocks;
    const uint32_t first = q * a.chunk;
    const int left = first < n ? static_cast<int>(n - first) : 0, count = left < a.chunk ? left : a.chunk;
    const uint32_t none = 0xFFFFFFFFu;
    const uint32_t prev = count > 0 && first > 0 ? a.sorted[first - 1].row : none;
    const uint32_t next = count > 0 && first + count < n ? a.sorted[first + count].row : none;
    // a wavefront keeps its chunk's pairs in its lanes, smaller groups in LDS
    Pair own = {0u, 0u};
    Pair* mine = pairs + (kWave ? 0 : g * a.chunk);
    if constexpr (kWave) {
        if (lane < count) own = a.sorted[first + lane];
    } else {
        for (int i = lane; i < count; i += a.lanes) mine[i] = a.sorted[first + i];
        __syncthreads();
    }
    auto row_of = [&](int i) -> uint32_t {
        if constexpr (kWave)
            return __builtin_amdgcn_readlane(own.row, i);
        else
            return mine[i].row;
    };
    auto token_of = [&](int i) -> uint32_t {
        if constexpr (kWave)
            return __builtin_amdgcn_readlane(own.token, i);
        else
            return mine[i].token;
    };
    const int64_t c = (static_cast<int64_t>(col) * a.lanes + lane) * kV;
    if (count == 0 || (!kWave && c >= a.cols)) return;
    const bool there = c < a.cols;
    float acc[kV] = {};
    uint32_t cur = row_of(0);
    bool before = cur == prev;
    auto flush = [&](bool on) {
        if (!there) return;
        if (before || on) {
            float* p = a.partial + (2 * static_cast<int64_t>(q) + (before ? 0 : 1)) * a.wide + c;
#pragma unroll
            for (int k = 0; k < kV; k += 4)
                *reinterpret_cast<u32x4*>(p + k) = (u32x4){__float_as_uint(acc[k]), __float_as_uint(acc[k + 1]),
                                                           __float_as_uint(acc[k + 2]), __float_as_uint(acc[k + 3])};
        } else {
            finish_row<kV>(a, cur, c, acc, kAdd);
        }
    };
    Piece<kS, kV> x[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
        if (u < count) x[u].template load<true>(a.src + token_of(u) * a.src_stride, c, a.cols);
    for (int i = 0; i < count; i += kAhead) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (i + u >= count) break;
            const uint32_t row = row_of(i + u);
            if (row != cur) {
                flush(false);
                cur = row;
                before = false;
#pragma unroll
                for (int k = 0; k < kV; ++k) acc[k] = 0.0f;
            }
#pragma unroll
            for (int k = 0; k < kV; ++k) acc[k] += x[u][k];
            if (i + u + kAhead < count)
                x[u].template load<true>(a.src + token_of(i + u + kAhead) * a.src_stride, c, a.cols);
        }
    }
    flush(cur == next);
}

// Rows that go on from one chunk into others: by the group of the chunk in
// which the row begins, the partials in order.  A row that has many chunks is
// one group's, kJoinAhead loads at a time: 131072 x 4096 fp16, by text's law 284
// us in all, with half of the tokens on one id 314.
constexpr int kJoinCols = 4;
constexpr int kJoinAhead = 16;

__global__ __launch_bounds__(kThreads) void join_kernel(GradArgs a) {
    const int lane = threadIdx.x & (a.lanes - 1);
    const uint32_t block = blockIdx.x / a.col_blocks, col = blockIdx.x - block * a.col_blocks;
    const uint32_t n = a.heads[0], chunk = a.chunk;
    const uint32_t q = block * (kThreads / a.lanes) + threadIdx.x / a.lanes, first = q * chunk, end = first + chunk;
    if (first >= n || end >= n) return;
    const uint32_t row = a.sorted[end - 1].row;
    if (a.sorted[end].row != row) return;
    if (first > 0 && a.sorted[first - 1].row == row) return;  // begins before
    // the last chunk that has this row: it goes on into those whose first token has it
    const uint32_t chunks = (n + chunk - 1) / chunk;
    const uint64_t group = (a.lanes == 64 ? ~uint64_t{0} : (uint64_t{1} << a.lanes) - 1)
                           << ((threadIdx.x & 63) / a.lanes * a.lanes);
    uint32_t last = q + 1;
    while (true) {
        const uint32_t k = last + 1 + lane;
        const bool on = k < chunks && a.sorted[k * chunk].row == row;
        const int more = __popcll(__ballot(on) & group);
        last += more;
        if (more < a.lanes) break;
    }
    const int64_t c = (static_cast<int64_t>(col) * a.lanes + lane) * kJoinCols;
    if (c >= a.cols) return;
    const uint8_t* p = reinterpret_cast<const uint8_t*>(a.partial + c);
    const int64_t bytes = a.wide * static_cast<int64_t>(sizeof(float));
    Piece<kFP32, kJoinCols> x[kJoinAhead];
    x[0].load<false>(p + (2 * static_cast<int64_t>(q) + 1) * bytes, 0, kJoinCols);
    float acc[kJoinCols];
#pragma unroll
    for (int k = 0; k < kJoinCols; ++k) acc[k] = x[0][k];
    for (uint32_t j = q + 1; j <= last; j += kJoinAhead) {
#pragma unroll
        for (int u = 0; u < kJoinAhead; ++u)
            x[u].load<false>(p + 2 * static_cast<int64_t>(j + u < last ? j + u : last) * bytes, 0, kJoinCols);
#pragma unroll
        for (int u = 0; u < kJoinAhead; ++u)
            if (j + u <= last)
#pragma unroll
                for (int k = 0; k < kJoinCols; ++k) acc[k] += x[u][k];
    }
    finish_row<kJoinCols>(a, row, c, acc, a.accumulate != 0);
}

// ---- host --------------------------------------------------------------------

constexpr int64_t kMaxRows = int64_t{1} << 22;  // two radix passes of kMaxDigits
constexpr int64_t kMaxTokens = INT32_MAX;
constexpr int64_t kMaxCols = int64_t{1} << 24;
constexpr int64_t kMaxGrid = int64_t{1} << 24;  // blocks of kThreads that a launch can have

// Lanes of a row: the power of two from `least` to `most` that one column block
// needs, or, where it takes several, down to `down_to`, the one with the fewest
// idle lanes over all of them, the larger one of equals.
int lanes_for(int64_t cols, int per_lane, int least, int most, int down_to) {
    const int64_t need = (cols + per_lane - 1) / per_lane;
    int lanes = least;
    while (lanes < most && lanes < need) lanes *= 2;
    if (need > lanes) {
        int64_t best = (need + lanes - 1) / lanes * lanes;
        for (int l = lanes / 2; l >= down_to; l /= 2) {
            const int64_t all = (need + l - 1) / l * l;
            if (all < best) {
                best = all;
                lanes = l;
            }
        }
    }
    return lanes;
}

uint32_t col_blocks(int64_t cols, int per_lane, int lanes) {
    return static_cast<uint32_t>((cols + int64_t{per_lane} * lanes - 1) / (int64_t{per_lane} * lanes));
}

// The form of one gradient call and the parts of its workspace.
struct GradPlan {
    bool direct, bucket;
    int key_bits, bucket_bits, passes, sort_blocks, sort_tokens, chunk;
    int64_t chunks;
    size_t heads, counts, first, sorted, partial, bytes;
};

GradPlan plan_grad(int64_t tokens, int64_t rows, int64_t cols) {
    GradPlan p{};
    p.direct = tokens <= kDirectTokens;
    if (p.direct) return p;
    while (int64_t{1} << p.key_bits < rows) ++p.key_bits;
    p.passes = int64_t{1} << p.key_bits <= kMaxDigits ? 1 : 2;
    // rows of a bucket: 256 buckets, of 16 rows at least
    while (p.bucket_bits < 4 || rows >> p.bucket_bits > 256) ++p.bucket_bits;
    p.bucket = tokens <= kBucketTokens && 1 << p.bucket_bits <= kBucketDigits;
    int64_t per = (tokens + kMaxSortBlocks - 1) / kMaxSortBlocks;
    per = (per + kSortThreads - 1) / kSortThreads * kSortThreads;
    p.sort_tokens = static_cast<int>(per);
    p.sort_blocks = static_cast<int>((tokens + per - 1) / per);
    const int l = lanes_for(cols, 8, kMinLanes, 64, kMinLanes);
    const int64_t waves = tokens * col_blocks(cols, 8, l) * l / 64;
    // Longer chunks have fewer partials, shorter ones keep more loads in flight
    // (us with chunks of 16, 32 and 64, bf16, text's law: 2048 tokens into 1000 x
    // 256 17.8, 24, 38, 8192 into 50304 x 2048 60, 62, 75, 16384 76, 75, 80, 30000
    // into 20011 x 1001 64, 74, 95, 91000 into 883 x 640 -, 54, 65, 131072 into
    // 32000 x 4096 406, 377, 362, into 1000 x 64 61, 46, 46).
    p.chunk = waves >= 524288 ? 64 : waves >= 65536 || tokens > 65536 ? 32 : 16;
    p.chunks = (tokens + p.chunk - 1) / p.chunk;
    const int64_t wide = (cols + 7) / 8 * 8;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at = (at + bytes + 255) / 256 * 256;
        return here;
    };
    p.heads = take(sizeof(uint32_t));
    p.counts = take(p.bucket ? 0 : sizeof(uint32_t) * p.sort_blocks * kMaxDigits);
    p.first = take(p.bucket || p.passes == 1 ? 0 : sizeof(Pair) * tokens);
    p.sorted = take(sizeof(Pair) * tokens);
    p.partial = take(sizeof(float) * 2 * p.chunks * wide);
    p.bytes = at;
    return p;
}

int check_matrix(const char* name, const char* what, const gockpt_matrix* m) {
    if (m == nullptr) return ops_fail(GOCKPT_EINVAL, "%s: null %s", name, what);
    if (!dtype_ok(m->dtype)) return ops_fail(GOCKPT_EINVAL, "%s: %s dtype %d", name, what, m->dtype);
    if (m->rows < 0 || m->cols < 0 || m->rows > kMaxTokens || m->cols > kMaxCols)
        return ops_fail(GOCKPT_EINVAL, "%s: %s of %lld x %lld", name, what, static_cast<long long>(m->rows),
                        static_cast<long long>(m->cols));
    if (m->rows > 1 && (m->stride < m->cols || m->stride > (int64_t{1} << 46) / m->rows))
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
    ids->magic = t->length > 1 ? static_cast<uint32_t>((uint64_t{1} << 32) / t->length) : UINT32_MAX;
    return GOCKPT_OK;
}

// The output goes past the caches above this size.  us of a lookup and a kernel
// that reads its output, with plain and with nontemporal stores: 32 MiB 23.2
// and 24.1, 64 MiB 39.4 and 40.2, 128 MiB 80.9 and 80.1, 512 MiB 339 and 324.
constexpr int64_t kCachedOutBytes = int64_t{96} << 20;
template <int kW, int kO>
int launch_lookup(LookupArgs& a, const char* name, hipStream_t s) {
    constexpr int kV = kO == kFP32 ? 4 : 8;
    a.lanes = lanes_for(a.cols, kV, 1, kThreads, 64);
    a.col_blocks = col_blocks(a.cols, kV, a.lanes);
    const int64_t per = kThreads / a.lanes;
    const int64_t blocks = ((a.ids.tokens + per - 1) / per * a.col_blocks + kPieces - 1) / kPieces;
    if (blocks >= kMaxGrid) return ops_fail(GOCKPT_EINVAL, "%s: out is too large", name);
    const bool nt = a.ids.tokens * a.cols * dtype_bytes(kO) > kCachedOutBytes;
    hipLaunchKernelGGL((nt ? lookup_kernel<kW, kO, true> : lookup_kernel<kW, kO, false>),
                       dim3(static_cast<uint32_t>(blocks)), dim3(kThreads), 0, s, a);
    return ops_launched(name);
}

template <int kW>
int launch_lookup(LookupArgs& a, int out_dtype, const char* name, hipStream_t s) {
    if (out_dtype == kBF16) return launch_lookup<kW, kBF16>(a, name, s);
    if (out_dtype == kFP16) return launch_lookup<kW, kFP16>(a, name, s);
    return launch_lookup<kW, kFP32>(a, name, s);
}

// Sort launch number `part`: its blocks that sort, and those that clear the
// table.
dim3 sort_grid(GradArgs& a, int part) {
    a.part = part;
    return dim3(a.sort_blocks + (a.clear_from < a.ids.rows ? kClearBlocks : 0));
}

void launch_sort(GradArgs& a, const GradPlan& p, hipStream_t s) {
    if (p.bucket) {
        a.parts = 1;
        a.sort_blocks = static_cast<int>((int64_t{a.ids.rows} + (1 << p.bucket_bits) - 1) >> p.bucket_bits);
        hipLaunchKernelGGL(bucket_kernel, sort_grid(a, 0), dim3(kSortThreads), 0, s, a, p.bucket_bits);
        return;
    }
    a.sort_blocks = p.sort_blocks;
    a.sort_tokens = p.sort_tokens;
    a.parts = 2 * p.passes;
    const int low = p.passes == 2 ? (p.key_bits + 1) / 2 : p.key_bits;
    a.shift = 0;
    a.digits = 1 << low;
    hipLaunchKernelGGL(count_kernel<true>, sort_grid(a, 0), dim3(kSortThreads), 0, s, a);
    hipLaunchKernelGGL(place_kernel<true>, sort_grid(a, 1), dim3(kSortThreads), 0, s, a,
                       p.passes == 2 ? a.first : a.sorted);
    if (p.passes == 1) return;
    a.shift = low;
    a.digits = 1 << (p.key_bits - low);
    hipLaunchKernelGGL(count_kernel<false>, sort_grid(a, 2), dim3(kSortThreads), 0, s, a);
    hipLaunchKernelGGL(place_kernel<false>, sort_grid(a, 3), dim3(kSortThreads), 0, s, a, a.sorted);
}

template <int kS>
int launch_grad(GradArgs& a, const GradPlan& p, const char* name, hipStream_t s) {
    constexpr int kV = kS == kFP32 ? 4 : 8;
    if (p.direct) {
        a.lanes = lanes_for(a.cols, kV, 1, kThreads, 64);
        a.col_blocks = col_blocks(a.cols, kV, a.lanes);
        a.clear_nt = a.ids.rows * a.cols * dtype_bytes(a.dst_dtype) > kCachedOutBytes;
        const int64_t blocks = (int64_t{a.ids.rows} + kBucketRows - 1) / kBucketRows * a.col_blocks;
        if (blocks >= kMaxGrid) return ops_fail(GOCKPT_EINVAL, "%s: the table is too large", name);
        hipLaunchKernelGGL(direct_kernel<kS>, dim3(static_cast<uint32_t>(blocks)), dim3(kThreads), 0, s, a);
        return ops_launched(name);
    }
    // Whole wavefronts where there are few tokens (narrow rows then leave lanes
    // idle, but rows end together: 2304 x 77 23.6 us, 24.4 in groups of 16); with
    // many, the groups with the fewest idle lanes (102016 x 637 80, 100).
    const int least = p.bucket ? 64 : kMinLanes;
    a.lanes = lanes_for(a.cols, kV, least, 64, least);
    a.col_blocks = col_blocks(a.cols, kV, a.lanes);
    a.chunk = p.chunk;
    const int groups = kThreads / a.lanes;
    const int64_t blocks = (p.chunks * a.col_blocks + groups - 1) / groups;
    if (2 * blocks >= kMaxGrid) return ops_fail(GOCKPT_EINVAL, "%s: too many tokens", name);
    a.clear_from = a.ids.rows;
    a.sum_blocks = static_cast<uint32_t>(blocks);
    int64_t clear_blocks = 0;
    if (!a.accumulate) {
        const int64_t bytes = p.bucket ? kClearBucketBytes : 2 * p.passes * kClearRadixBytes;
        const int64_t row_bytes = a.cols * dtype_bytes(a.dst_dtype), early = bytes / row_bytes;
        a.clear_nt = a.clear_from * row_bytes > kCachedOutBytes;
        a.clear_from = early < a.clear_from ? a.clear_from - early : 0;
        clear_blocks = (a.clear_from + kClearRows - 1) / kClearRows;
    }
    launch_sort(a, p, s);
    const dim3 grid(static_cast<uint32_t>(blocks + clear_blocks));
    a.wide = (a.cols + 7) / 8 * 8;
    if (a.lanes == 64)
        hipLaunchKernelGGL((a.accumulate ? sum_kernel<kS, true, true> : sum_kernel<kS, true, false>), grid,
                           dim3(kThreads), 0, s, a);
    else
        hipLaunchKernelGGL((a.accumulate ? sum_kernel<kS, false, true> : sum_kernel<kS, false, false>), grid,
                           dim3(kThreads), 0, s, a);
    a.lanes = lanes_for(a.cols, kJoinCols, kMinLanes, 64, kMinLanes);
    a.col_blocks = col_blocks(a.cols, kJoinCols, a.lanes);
    const int64_t jblocks = (p.chunks + kThreads / a.lanes - 1) / (kThreads / a.lanes) * a.col_blocks;
    hipLaunchKernelGGL(join_kernel, dim3(static_cast<uint32_t>(jblocks)), dim3(kThreads), 0, s, a);
    return ops_launched(name);
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
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (table->dtype == kBF16) return launch_lookup<kBF16>(a, out->dtype, name, s);
    if (table->dtype == kFP16) return launch_lookup<kFP16>(a, out->dtype, name, s);
    return launch_lookup<kFP32>(a, out->dtype, name, s);
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
    // a single row may come with any stride; the kernels take rows whose stride
    // is their width as one span
    a.dst_stride = (grad_table->rows > 1 ? grad_table->stride : grad_table->cols) * dtype_bytes(grad_table->dtype);
    a.scale = scale;
    a.dst_dtype = grad_table->dtype;
    a.accumulate = accumulate != 0;
    hipStream_t s = static_cast<hipStream_t>(stream);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    a.heads = reinterpret_cast<uint32_t*>(ws + p.heads);
    a.counts = reinterpret_cast<uint32_t*>(ws + p.counts);
    a.first = reinterpret_cast<Pair*>(ws + p.first);
    a.sorted = reinterpret_cast<Pair*>(ws + p.sorted);
    a.partial = reinterpret_cast<float*>(ws + p.partial);
    if (grad_out->dtype == kBF16) return launch_grad<kBF16>(a, p, name, s);
    if (grad_out->dtype == kFP16) return launch_grad<kFP16>(a, p, name, s);
    return launch_grad<kFP32>(a, p, name, s);
}

}  // extern "C"
