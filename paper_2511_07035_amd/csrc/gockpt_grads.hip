// gockpt_grads.hip -- norm and clipping of a list of gradient tensors.
//
//   sumsq_kernel   reads every tensor once: S = sum of squares, one fp64
//                  partial a block; block 0 adds them in a fixed order:
//                  norm = sqrt(S) / scale, the clipping coefficient
//                  min(1, max_norm / (norm + 1e-6)), and found_inf: an inf or
//                  NaN, or a finite element whose scaled value is rounded to
//                  an infinity in a narrower type.
//   scale_kernel   element * coef, rounded to the destination's type.
//   whole_kernel   all of it in one launch for a list of at most 512 tiles.
//
// The host cuts the tensors into tiles of at most 1024 units of 16 source
// bytes (16 KiB) once, when the list is made; a tensor of any size, type,
// stride or start is a few entries of one table, and one launch covers all.
//
// Memory bounds all of it: 2 flops an element against 2 or 4 bytes read.  On
// the 1.31e9 bf16 gradients of GPT 1.3B (2.62 GB in 195 tensors) the norm takes
// 374 us, 7.0 TB/s, which is what a read-only probe reaches.  Clipping reads
// twice, since no element can be scaled before the last one is squared: 5.2 GB
// of fp32 gradients rounded into bf16 take 1995 us, 6.6 TB/s over the 13.1 GB
// moved; 2.6 GB of bf16 in place 1235, 6.4 TB/s over 7.9 GB.  In a small list a
// launch costs more than the data, hence whole_kernel.
#include <math.h>
#include <stdlib.h>

#include <new>
#include <vector>

#include "gockpt_ops_internal.h"

#pragma clang fp contract(off)

namespace gockpt {

namespace {

constexpr int kThreads = 256;
constexpr int kUnitsPerThread = 4;
constexpr int kTileUnits = kThreads * kUnitsPerThread;

// Blocks of sumsq_kernel.  Each keeps the next tile's loads in flight during
// the arithmetic of the current one, so 4 blocks a compute unit are enough and
// fewer partials are left to add (GPT 1.3B in bf16 376 us, with 2048 390).
constexpr int kSumBlocks = 1024;

// Lists of up to this many tiles (8 MiB where the tensors fill theirs; 512
// tensors of any size below) take one launch, a tile a block.  us a clip in one
// launch and in two: 2^17 bf16 elements 5.6 and 8.8, 2^21 7.1 and 9.7, 2^22, the
// limit, 10.1 and 11.0.  Above it, blocks of two or four tiles that keep them in
// registers gained nothing (2^23 16.3 and 16.2).
constexpr int kWholeTiles = 512;
// Polls (about 0.5 us each) before a block of whole_kernel computes the partials
// it misses, and before block 0 does, which in a large list is a lot of work for
// one block; none with GOCKPT_TEST_GRADS_AGAIN=1 in the environment when the list
// is made, with which tests reach that path.
constexpr int kWholeSpins = 64;
constexpr int kSpins0 = 1 << 20;

// Clipping up to this many source bytes: the sums leave what they read in the
// last-level cache, and scale_kernel, last tiles first, finds part of it there
// (us cached and with nontemporal loads: 1.3e8 bf16 elements 128 and 134,
// 2.7e8 256 and 260; 1.3e9 fp32 2086 and 1992).  The norm alone always reads
// with the hint (1.3e9 bf16 390 against 436).
constexpr int64_t kCachedSumBytes = int64_t{512} << 20;
// scale_kernel has the hint on loads and stores where it moves more than this
// (us without and with it: 64 MiB in and out 36.5 and 37.8, 128 MiB 79.7 and
// 68.1; fp32 to bf16 64 + 32 MiB 30.7 and 32.5, 128 + 64 MiB 63.0 and 56.2).
constexpr int64_t kCachedScaleBytes = int64_t{144} << 20;
constexpr double kClipEps = 1e-6;

// Rows of one tensor, or a piece of one row.  Unit u of a tile is unit u %
// per_row of row u / per_row.  A unit is 16 bytes of source; a row's last one
// is the 16 bytes that end with the row, of which the first `skip` belong to
// the unit before (or, in a row of under 16 bytes, to nothing).
struct GradTile {
    const uint8_t* src;
    uint8_t* dst;
    int64_t stride;    // bytes from a row to the next
    int64_t dst_row;   // the same in dst
    int32_t units;     // of the tile, at most kTileUnits
    int32_t per_row;   // units of a row
    uint32_t magic;    // per_row > 1: floor(2^32 / per_row) + 1, u / per_row is the high word of u * magic
    int16_t skip;      // of a row's last unit: 0 to 14
    int8_t dtype, dst_dtype;
};
static_assert(sizeof(GradTile) == 48, "table entry");

// u * magic >> 32 is u / d for every u <= kTileUnits: the product exceeds
// u * 2^32 / d by at most u, and u * d <= kTileUnits^2 < 2^32.
__device__ __forceinline__ void unit_place(const GradTile& t, uint32_t u, uint32_t& row, uint32_t& k) {
    if (t.units == t.per_row) {
        row = 0;
        k = u;
    } else if (t.per_row == 1) {
        row = u;
        k = 0;
    } else {
        row = __umulhi(u, t.magic);
        k = u - row * static_cast<uint32_t>(t.per_row);
    }
}

__device__ __forceinline__ uint32_t unit_skip(const GradTile& t, uint32_t k) {
    return k + 1 == static_cast<uint32_t>(t.per_row) ? t.skip : 0;
}

// The units of this thread, zeros beyond the tile's end.  What a last unit
// skips is not cleared: that would wait for the load.
template <bool kNT>
__device__ __forceinline__ void load_tile(const GradTile& t, u32x4 (&raw)[kUnitsPerThread]) {
    if (t.per_row == 1 && t.skip > 0) {  // rows of under 16 bytes
#pragma unroll
        for (int i = 0; i < kUnitsPerThread; ++i) {
            const uint32_t u = i * kThreads + threadIdx.x;
            raw[i] = (u32x4){0u, 0u, 0u, 0u};
            if (u >= static_cast<uint32_t>(t.units)) continue;
            const uint16_t* h = reinterpret_cast<const uint16_t*>(t.src + u * t.stride - t.skip);
#pragma unroll
            for (int j = 1; j < 8; ++j)
                if (2 * j >= t.skip) raw[i][j / 2] |= static_cast<uint32_t>(h[j]) << (16 * (j & 1));
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < kUnitsPerThread; ++i) {
        const uint32_t u = i * kThreads + threadIdx.x;
        raw[i] = (u32x4){0u, 0u, 0u, 0u};
        if (u >= static_cast<uint32_t>(t.units)) continue;
        uint32_t row, k;
        unit_place(t, u, row, k);
        const u32x4_any* p =
            reinterpret_cast<const u32x4_any*>(t.src + row * t.stride + k * 16u - unit_skip(t, k));
        raw[i] = kNT ? __builtin_nontemporal_load(p) : *p;
    }
}

// Clears what a tile's last units skip.
__device__ __forceinline__ void clear_skipped(const GradTile& t, u32x4 (&raw)[kUnitsPerThread]) {
    if (t.skip == 0) return;
#pragma unroll
    for (int i = 0; i < kUnitsPerThread; ++i) {
        uint32_t row, k;
        unit_place(t, i * kThreads + threadIdx.x, row, k);
        const int skip = static_cast<int>(unit_skip(t, k));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (skip >= 4 * j + 2) raw[i][j] &= 0xFFFF0000u;
            if (skip >= 4 * j + 4) raw[i][j] = 0u;
        }
    }
}

template <int kT, class F>
__device__ __forceinline__ void each_elem(u32x4 raw, F&& f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (kT == kFP32) {
            f(__uint_as_float(raw[i]));
        } else {
            f(elem_to_f32<kT>(raw[i] & 0xFFFFu));
            f(elem_to_f32<kT>(raw[i] >> 16));
        }
    }
}

// Sum of squares of a thread's units (at most 32 elements).  In fp32 unless
// that may have lost something: an fp32 sum in [2^-100, 2^126) has overflowed
// nowhere, and what its terms lost below 2^-149 is under 2^-44 of it.  (All in
// fp64 would be two more operations an element at a lower rate.)
// Otherwise (or where it is NaN), and if some element is not zero, the squares
// are added again in fp64, where those of fp32 values neither overflow nor
// vanish and the sum is finite exactly when every element is.
template <int kT>
__device__ __forceinline__ double square_sum(const u32x4 (&raw)[kUnitsPerThread]) {
    float s = 0.0f;
    uint32_t any = 0u;
#pragma unroll
    for (int i = 0; i < kUnitsPerThread; ++i) {
        any |= raw[i][0] | raw[i][1] | raw[i][2] | raw[i][3];
        each_elem<kT>(raw[i], [&](float x) { s = __builtin_fmaf(x, x, s); });
    }
    if ((s >= 0x1p-100f && s < 0x1p126f) || any == 0u) return static_cast<double>(s);
    double d = 0.0;
#pragma unroll
    for (int i = 0; i < kUnitsPerThread; ++i)
        each_elem<kT>(raw[i], [&](float x) { d = __builtin_fma(static_cast<double>(x), static_cast<double>(x), d); });
    return d;
}

// The sum over the block, and bits 0 and 1 of `flags` or'ed over it.
__device__ __forceinline__ double block_sum(double x, uint32_t& flags) {
    __shared__ double part[kThreads / 64];
    __shared__ uint32_t bits[kThreads / 64];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
    const uint32_t f = (__ballot(flags & 1u) != 0u ? 1u : 0u) | (__ballot(flags & 2u) != 0u ? 2u : 0u);
    __syncthreads();  // an earlier sum has been read
    if ((threadIdx.x & 63) == 0) {
        part[threadIdx.x >> 6] = x;
        bits[threadIdx.x >> 6] = f;
    }
    __syncthreads();
    flags = bits[0] | bits[1] | bits[2] | bits[3];
    return (part[0] + part[1]) + (part[2] + part[3]);
}

// The least fp32 magnitudes that round to an infinity: half a step above the
// type's largest finite value, where the tie goes to the even side, upwards.
constexpr float kInfOfFp16 = 65520.0f;
constexpr float kInfOfBf16 = 0x1.FFp127f;

// Largest magnitudes of the elements that go to fp16 from a wider type and are
// too large for it as they are, and of such that go to bf16 from fp32, as the
// bits of an fp32 value, which order as the values do (0: none; an infinity or
// NaN lies above all).  Whether one of them is still rounded to infinity is
// known once the coefficient is (at most 1): the products with it order as the
// elements do.
struct Range {
    uint32_t fp16, bf16;
};

__device__ __forceinline__ uint32_t max_bits(uint32_t a, uint32_t b) { return a > b ? a : b; }

// raw, whose squares' sum is `sum`, into range.  An element of least magnitude
// x makes the sum x^2 (1 - 2^-24) at least, so almost always the sum alone tells
// that there is none.
__device__ __forceinline__ void tile_range(const GradTile& t, const u32x4 (&raw)[kUnitsPerThread], double sum,
                                           Range& range) {
    const bool to16 = t.dst_dtype == kFP16 && t.dtype != kFP16;
    if (!to16 && !(t.dst_dtype == kBF16 && t.dtype == kFP32)) return;
    const float least = to16 ? kInfOfFp16 : kInfOfBf16;
    if (!(sum >= 0.5 * least * least)) return;  // a NaN among them: found without this
    const uint32_t mask = t.dtype == kBF16 ? 0x7FFF0000u : 0x7FFFFFFFu;
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < kUnitsPerThread; ++i) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            m = max_bits(m, raw[i][j] & mask);
            if (t.dtype == kBF16) m = max_bits(m, raw[i][j] << 16 & mask);
        }
    }
    if (m < __float_as_uint(least)) return;
    if (to16)
        range.fp16 = max_bits(range.fp16, m);
    else
        range.bf16 = max_bits(range.bf16, m);
}

__device__ __forceinline__ Range block_range(Range x) {
    __shared__ Range part[kThreads / 64];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        x.fp16 = max_bits(x.fp16, __shfl_xor(x.fp16, o, 64));
        x.bf16 = max_bits(x.bf16, __shfl_xor(x.bf16, o, 64));
    }
    __syncthreads();  // an earlier range has been read
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kThreads / 64; ++k) {
        x.fp16 = max_bits(x.fp16, part[k].fp16);
        x.bf16 = max_bits(x.bf16, part[k].bf16);
    }
    return x;
}

// raw -> the sum of its squares.
__device__ __forceinline__ double tile_sum(const GradTile& t, u32x4 (&raw)[kUnitsPerThread]) {
    clear_skipped(t, raw);
    if (t.dtype == kBF16) return square_sum<kBF16>(raw);
    if (t.dtype == kFP16) return square_sum<kFP16>(raw);
    return square_sum<kFP32>(raw);
}

// ---- exchange of the blocks' partials ------------------------------------------
//
// A partial is one 64-bit word: a double without its three lowest bits, in whose
// place are the call's epoch modulo four, the tag, and kSlotRange.  Every call on
// a list writes every slot, so a slot with the running call's tag is of this
// call: value and flag are one word, and no fence is needed, which on this chip
// would write back an XCD's L2.  In a list with destinations narrower than their
// source (kRange) a block writes its range too, as two magnitudes of 31 bits
// above the tag; kSlotRange says whether there is one to be read, since a second
// read of words costs 1 us.  Block 0 adds the partials in a fixed order and
// writes the result.  (As a launch of its own that cost 1 us more, with 2^23 and
// with 2^25 bf16 elements.)
//
// A block arrives when it has read the epoch, and the epoch is the number of
// arrivals, kGroupBlocks a call, divided by that: the next one is not reached
// before all blocks have read this one.  The blocks count in groups, each with a
// word and so an epoch of its own, the same in all between calls (arrivals at one
// word took 6 us for 1024 blocks).  No wait is without end: a block that has
// polled `spins` times computes the partials that it misses.  Calls on one list
// whose order the caller has not seen to therefore still end, with whatever
// results, and leave the list in order: their arrivals add up, and the tags that
// they leave behind are not that of the next call (of up to three such calls).

constexpr int kGroups = 64;
constexpr int kGroupBlocks = kSumBlocks / kGroups;  // at most
constexpr int kGroupWords = 32;                     // from a group's word to the next

constexpr uint64_t kSlotTag = 3;
constexpr uint64_t kSlotRange = 4;

__device__ __forceinline__ uint64_t slot_tag(uint32_t epoch) { return epoch & 3u; }

__device__ __forceinline__ uint64_t read_slot(const uint64_t* p) {
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__device__ __forceinline__ double slot_value(uint64_t word) {
    return __builtin_bit_cast(double, word & ~(kSlotTag | kSlotRange));
}

__device__ __forceinline__ uint64_t sum_word(double x, bool has_range, uint32_t epoch) {
    return (__builtin_bit_cast(uint64_t, x) & ~(kSlotTag | kSlotRange)) | (has_range ? kSlotRange : 0u) |
           slot_tag(epoch);
}

__device__ __forceinline__ uint64_t range_word(Range x, uint32_t epoch) {
    return uint64_t{x.fp16} << 33 | uint64_t{x.bf16} << 2 | slot_tag(epoch);
}

__device__ __forceinline__ void publish(uint64_t* slot, uint32_t epoch, double x, bool has_range) {
    __hip_atomic_store(slot, sum_word(x, has_range, epoch), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__device__ __forceinline__ void publish(uint64_t* slot, uint32_t epoch, Range x) {
    __hip_atomic_store(slot, range_word(x, epoch), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// This thread's slots, i, i + kThreads and so on below `blocks`; true while one
// is not of this epoch.
template <int kPer>
__device__ __forceinline__ bool read_slots(const uint64_t* slots, int blocks, uint32_t epoch, uint64_t (&word)[kPer]) {
    bool missing = false;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        const int b = k * kThreads + static_cast<int>(threadIdx.x);
        word[k] = b < blocks ? read_slot(slots + b) : slot_tag(epoch);
        missing |= (word[k] & kSlotTag) != slot_tag(epoch);
    }
    return missing;
}

// This thread's words of all blocks, after at most `spins` polls; true while one
// is not of this epoch.
template <int kPer>
__device__ __forceinline__ bool poll_slots(const uint64_t* slots, int blocks, uint32_t epoch, int spins,
                                           uint64_t (&word)[kPer]) {
    bool wait = read_slots(slots, blocks, epoch, word);
    for (int i = 0; wait && i < spins; ++i) {
        __builtin_amdgcn_s_sleep(2);
        wait = read_slots(slots, blocks, epoch, word);
    }
    return wait;
}

// Those words that are not of this epoch are computed: again(b) is block b's, by
// the whole block.
template <int kPer, class Again>
__device__ __forceinline__ void fill_words(const uint64_t* slots, int blocks, uint32_t epoch, uint64_t (&word)[kPer],
                                           Again&& again) {
    __shared__ uint64_t all[kPer * kThreads];
#pragma unroll
    for (int k = 0; k < kPer; ++k) all[k * kThreads + threadIdx.x] = word[k];
    __syncthreads();
    for (int b = 0; b < blocks; ++b) {
        if ((all[b] & kSlotTag) == slot_tag(epoch)) continue;  // the same for all threads
        const uint64_t w = again(b);
        if (threadIdx.x == 0) {
            const uint64_t now = read_slot(slots + b);
            all[b] = (now & kSlotTag) == slot_tag(epoch) ? now : w;
        }
        __syncthreads();
    }
#pragma unroll
    for (int k = 0; k < kPer; ++k) word[k] = all[k * kThreads + threadIdx.x];
}

// Block b's share of the tiles, every `step`-th from b on: the sum of their
// squares and their range, in the order in which block b takes them.  Tiles that
// may be scaled in place meanwhile go to their own type, so have no range.
template <bool kRange>
__device__ __forceinline__ double share_again(const GradTile* __restrict__ tiles, int ntiles, int b, int step,
                                              Range& range, bool& has_range) {
    double acc = 0.0;
    range = {0u, 0u};
    for (int i = b; i < ntiles; i += step) {
        const GradTile t = tiles[i];
        u32x4 raw[kUnitsPerThread];
        load_tile<false>(t, raw);
        const double sum = tile_sum(t, raw);
        acc += sum;
        if constexpr (kRange) tile_range(t, raw, sum, range);
    }
    uint32_t flags = kRange && (range.fp16 | range.bf16) != 0u;
    acc = block_sum(acc, flags);
    has_range = flags != 0u;
    if (has_range) range = block_range(range);
    return acc;
}

// The sum over all blocks' partials, in a fixed order, and whether one has a
// range.  By a whole block.
template <int kPer, bool kRange>
__device__ __forceinline__ double all_sums(const GradTile* __restrict__ tiles, int ntiles, const uint64_t* slots,
                                           uint32_t epoch, int spins, bool& has_range) {
    uint64_t word[kPer];
    const int blocks = gridDim.x;
    // bit 0: there is a range, bit 1: a word is missing
    uint32_t flags = poll_slots(slots, blocks, epoch, spins, word) ? 2u : 0u;
    auto sum = [&]() {
        double acc = 0.0;
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            acc += slot_value(word[k]);
            if (kRange && (word[k] & kSlotRange) != 0u) flags |= 1u;
        }
        return block_sum(acc, flags);
    };
    double acc = sum();
    if (flags & 2u) {
        fill_words(slots, blocks, epoch, word, [&](int b) {
            Range range;
            bool has;
            const double x = share_again<kRange>(tiles, ntiles, b, blocks, range, has);
            return sum_word(x, has, epoch);
        });
        flags = 0u;
        acc = sum();
    }
    has_range = flags != 0u;
    return acc;
}

// The range over all blocks.
template <int kPer>
__device__ __forceinline__ Range all_ranges(const GradTile* __restrict__ tiles, int ntiles, const uint64_t* ranges,
                                            uint32_t epoch, int spins) {
    uint64_t word[kPer];
    const int blocks = gridDim.x;
    if (__syncthreads_or(poll_slots(ranges, blocks, epoch, spins, word)))
        fill_words(ranges, blocks, epoch, word, [&](int b) {
            Range range;
            bool has;
            share_again<true>(tiles, ntiles, b, blocks, range, has);
            return range_word(range, epoch);
        });
    Range x = {0u, 0u};
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        x.fp16 = max_bits(x.fp16, static_cast<uint32_t>(word[k] >> 33));
        x.bf16 = max_bits(x.bf16, static_cast<uint32_t>(word[k] >> 2) & 0x7FFFFFFFu);
    }
    return block_range(x);
}

__device__ __forceinline__ uint32_t* arrivals_of(uint32_t* sync) {
    return sync + blockIdx.x % kGroups * kGroupWords;
}

// By thread 0 alone: the others have the epoch through LDS, where it is by the
// time that the block arrives.
__device__ __forceinline__ uint32_t read_arrivals(uint32_t* sync) {
    return __hip_atomic_load(arrivals_of(sync), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// This block has read the epoch.  A group's first block arrives for those it lacks.
__device__ __forceinline__ void arrive(uint32_t* sync) {
    const uint32_t others = (gridDim.x - 1u - blockIdx.x) / kGroups;
    __hip_atomic_fetch_add(arrivals_of(sync), blockIdx.x < kGroups ? kGroupBlocks - others : 1u, __ATOMIC_RELAXED,
                           __HIP_MEMORY_SCOPE_AGENT);
}

__device__ __forceinline__ void finish_result(double sumsq, Range range, const float* scale, double max_norm,
                                              gockpt_grad_result* out) {
    const double norm = sqrt(sumsq) / (scale != nullptr ? static_cast<double>(*scale) : 1.0);
    const bool finite = isfinite(sumsq);
    const double coef = max_norm / (norm + kClipEps);
    const float c = finite && coef < 1.0 ? static_cast<float>(coef) : 1.0f;
    const float fp16 = __uint_as_float(range.fp16), bf16 = __uint_as_float(range.bf16);
    out->sumsq = sumsq;
    out->norm = static_cast<float>(norm);
    out->found_inf = finite && fp16 * c < kInfOfFp16 && bf16 * c < kInfOfBf16 ? 0.0f : 1.0f;
    out->coef = c;
    out->reserved_[0] = fp16;
    out->reserved_[1] = bf16;
    out->reserved_[2] = 0.0f;
}

// Block 0 waits for the others, none of which waits for anything.
template <bool kNT, bool kRange>
__global__ __launch_bounds__(kThreads) void sumsq_kernel(const GradTile* __restrict__ tiles, int ntiles,
                                                         uint32_t* sync, uint64_t* slots, uint64_t* ranges,
                                                         int spins,
                                                         const float* __restrict__ scale, double max_norm,
                                                         gockpt_grad_result* __restrict__ out) {
    __shared__ uint32_t call;
    const uint32_t arrivals = threadIdx.x == 0 ? read_arrivals(sync) : 0u;
    double acc = 0.0;
    Range range = {0u, 0u};
    u32x4 next[kUnitsPerThread];
    int i = blockIdx.x;
    GradTile t = tiles[i];
    load_tile<kNT>(t, next);
    while (i < ntiles) {
        u32x4 raw[kUnitsPerThread];
#pragma unroll
        for (int k = 0; k < kUnitsPerThread; ++k) raw[k] = next[k];
        const GradTile now = t;
        i += gridDim.x;
        if (i < ntiles) {
            t = tiles[i];
            load_tile<kNT>(t, next);
        }
        const double sum = tile_sum(now, raw);
        acc += sum;
        if constexpr (kRange) tile_range(now, raw, sum, range);
    }
    uint32_t flags = kRange && (range.fp16 | range.bf16) != 0u;
    if (threadIdx.x == 0) call = arrivals / kGroupBlocks;
    acc = block_sum(acc, flags);
    bool has_range = flags != 0u;
    const uint32_t epoch = call;
    if (has_range) range = block_range(range);
    if (threadIdx.x == 0) {
        publish(slots + blockIdx.x, epoch, acc, has_range);
        if constexpr (kRange) publish(ranges + blockIdx.x, epoch, range);
        arrive(sync);
    }
    if (blockIdx.x != 0) return;
    constexpr int kPer = kSumBlocks / kThreads;
    acc = all_sums<kPer, kRange>(tiles, ntiles, slots, epoch, spins, has_range);
    if (has_range) range = all_ranges<kPer>(tiles, ntiles, ranges, epoch, spins);
    if (threadIdx.x == 0) finish_result(acc, range, scale, max_norm, out);
}

// The result of an empty list, or again from its sumsq and range.
__global__ void result_kernel(gockpt_grad_result* out, const float* scale, double max_norm, bool empty) {
    Range range = {0u, 0u};
    if (!empty) range = {__float_as_uint(out->reserved_[0]), __float_as_uint(out->reserved_[1])};
    finish_result(empty ? 0.0 : out->sumsq, range, scale, max_norm, out);
}

// One element, or two, four or eight, at any address.
template <int kT, int kN, bool kNT>
__device__ __forceinline__ void store_n(uint8_t* p, const float* x) {
    if constexpr (kT == kFP32) {
        if constexpr (kN > 4) {
            store_n<kT, 4, kNT>(p, x);
            store_n<kT, kN - 4, kNT>(p + 16, x + 4);
        } else {
            typedef float vec __attribute__((ext_vector_type(kN)));
            typedef vec vec_any __attribute__((aligned(2)));
            vec v;
#pragma unroll
            for (int i = 0; i < kN; ++i) {
                if constexpr (kN == 1)
                    v = x[i];
                else
                    v[i] = x[i];
            }
            if constexpr (kNT)
                __builtin_nontemporal_store(v, reinterpret_cast<vec_any*>(p));
            else
                *reinterpret_cast<vec_any*>(p) = v;
        }
    } else if constexpr (kN == 1) {
        store_elem<kT>(p, x[0]);
    } else {
        typedef uint32_t vec __attribute__((ext_vector_type(kN / 2)));
        typedef vec vec_any __attribute__((aligned(2)));
        vec v;
#pragma unroll
        for (int i = 0; i < kN / 2; ++i) {
            if constexpr (kN == 2)
                v = pack2<kT>(x[0], x[1]);
            else
                v[i] = pack2<kT>(x[2 * i], x[2 * i + 1]);
        }
        if constexpr (kNT)
            __builtin_nontemporal_store(v, reinterpret_cast<vec_any*>(p));
        else
            *reinterpret_cast<vec_any*>(p) = v;
    }
}

// One unit times coef to its place in dst (d: of its first byte, skipped or
// not).
template <int kS, int kD, bool kNT>
__device__ __forceinline__ void scale_unit(u32x4 raw, float coef, uint8_t* d, uint32_t skip) {
    constexpr int kN = kS == kFP32 ? 4 : 8;
    constexpr int kB = kD == kFP32 ? 4 : 2;
    float x[kN];
    int n = 0;
    each_elem<kS>(raw, [&](float v) { x[n++] = v * coef; });
    if (skip == 0) {
        store_n<kD, kN, kNT>(d, x);
    } else {
        const int from = skip / (kS == kFP32 ? 4 : 2);
#pragma unroll
        for (int i = 1; i < kN; ++i)
            if (i >= from) store_elem<kD>(d + kB * i, x[i]);
    }
}

template <int kS, int kD, bool kNT>
__device__ __forceinline__ void scale_units(const GradTile& t, const u32x4 (&raw)[kUnitsPerThread], float coef) {
#pragma unroll
    for (int i = 0; i < kUnitsPerThread; ++i) {
        const uint32_t u = i * kThreads + threadIdx.x;
        if (u >= static_cast<uint32_t>(t.units)) break;
        uint32_t row, k;
        unit_place(t, u, row, k);
        constexpr int kSrcBytes = kS == kFP32 ? 4 : 2, kDstBytes = kD == kFP32 ? 4 : 2;
        const int skip = static_cast<int>(unit_skip(t, k));
        const int at = (static_cast<int>(k) * 16 - skip) / kSrcBytes * kDstBytes;
        scale_unit<kS, kD, kNT>(raw[i], coef, t.dst + row * t.dst_row + at, skip);
    }
}

// raw * coef to the tile's places in dst.
template <bool kNT>
__device__ __forceinline__ void scale_tile(const GradTile& t, const u32x4 (&raw)[kUnitsPerThread], float coef) {
    if (t.dst == t.src && coef == 1.0f) return;
    switch (t.dtype * 3 + t.dst_dtype) {
        case kBF16 * 3 + kBF16: scale_units<kBF16, kBF16, kNT>(t, raw, coef); break;
        case kBF16 * 3 + kFP16: scale_units<kBF16, kFP16, kNT>(t, raw, coef); break;
        case kBF16 * 3 + kFP32: scale_units<kBF16, kFP32, kNT>(t, raw, coef); break;
        case kFP16 * 3 + kBF16: scale_units<kFP16, kBF16, kNT>(t, raw, coef); break;
        case kFP16 * 3 + kFP16: scale_units<kFP16, kFP16, kNT>(t, raw, coef); break;
        case kFP16 * 3 + kFP32: scale_units<kFP16, kFP32, kNT>(t, raw, coef); break;
        case kFP32 * 3 + kBF16: scale_units<kFP32, kBF16, kNT>(t, raw, coef); break;
        case kFP32 * 3 + kFP16: scale_units<kFP32, kFP16, kNT>(t, raw, coef); break;
        default: scale_units<kFP32, kFP32, kNT>(t, raw, coef); break;
    }
}

// One tile a block, the last tiles first (sumsq_kernel read them last).  A
// launch of all tiles is faster than 2048 blocks that walk over them: 1.3e9
// fp32 elements into bf16 2145 us a clip against 2292.
template <bool kNT>
__global__ __launch_bounds__(kThreads) void scale_kernel(const GradTile* __restrict__ tiles, int ntiles,
                                                         const gockpt_grad_result* __restrict__ result) {
    const float coef = result->coef;
    const GradTile t = tiles[ntiles - 1 - static_cast<int>(blockIdx.x)];
    if (t.dst == t.src && coef == 1.0f) return;
    u32x4 raw[kUnitsPerThread];
    load_tile<kNT>(t, raw);
    scale_tile<kNT>(t, raw, coef);
}

// ---- small lists: one launch ---------------------------------------------------
//
// Block b squares tile b, publishes its partial and, to clip, waits for the
// partials of all blocks, adds them in the order that every block uses, and
// scales the tile, which it still has in registers.  For a norm only block 0
// waits.
//
// A block that misses a partial after its polls computes it.  That tile may be
// scaled in place by its owner while it is read here, but the owner scales only
// after it has seen its own partial published: if the slot is still empty after
// the tile has been read, what was read is unscaled, and if it is not, the
// slot's value is taken.

template <bool kClip, bool kRange>
__global__ __launch_bounds__(kThreads) void whole_kernel(const GradTile* __restrict__ tiles, uint32_t* sync,
                                                         uint64_t* slots, uint64_t* ranges, int spins, int spins0,
                                                         const float* __restrict__ scale, double max_norm,
                                                         gockpt_grad_result* __restrict__ out) {
    __shared__ uint32_t call;
    __shared__ float coef;
    const uint32_t arrivals = threadIdx.x == 0 ? read_arrivals(sync) : 0u;
    const GradTile t = tiles[blockIdx.x];
    u32x4 raw[kUnitsPerThread];
    load_tile<false>(t, raw);
    const double sum = tile_sum(t, raw);
    Range range = {0u, 0u};
    if constexpr (kRange) tile_range(t, raw, sum, range);
    uint32_t flags = kRange && (range.fp16 | range.bf16) != 0u;
    if (threadIdx.x == 0) call = arrivals / kGroupBlocks;
    const double mine = block_sum(sum, flags);
    bool has_range = flags != 0u;
    const uint32_t epoch = call;
    if (has_range) range = block_range(range);
    if (threadIdx.x == 0) {
        publish(slots + blockIdx.x, epoch, mine, has_range);
        if constexpr (kRange) publish(ranges + blockIdx.x, epoch, range);
        arrive(sync);
    }
    if (!kClip && blockIdx.x != 0) return;

    constexpr int kPer = kWholeTiles / kThreads;
    const int polls = blockIdx.x == 0 ? spins0 : spins;
    const double acc = all_sums<kPer, kRange>(tiles, gridDim.x, slots, epoch, polls, has_range);
    // the coefficient does not depend on it, so only the block that writes the result needs it
    if (has_range && blockIdx.x == 0) range = all_ranges<kPer>(tiles, gridDim.x, ranges, epoch, polls);
    if (threadIdx.x == 0) {
        gockpt_grad_result r;
        finish_result(acc, range, scale, max_norm, &r);
        coef = r.coef;
        if (blockIdx.x == 0) *out = r;
    }
    if constexpr (kClip) {
        __syncthreads();
        scale_tile<false>(t, raw, coef);
    }
}

// ---- host: the table ---------------------------------------------------------

constexpr int64_t kMaxElems = int64_t{1} << 46;
// Workspace: arrivals, the blocks' partials, their ranges, table.
constexpr size_t kSlotsOff = kGroups * kGroupWords * sizeof(uint32_t);
constexpr size_t kRangesOff = kSlotsOff + kSumBlocks * sizeof(uint64_t);
constexpr size_t kTableOff = kRangesOff + kSumBlocks * sizeof(uint64_t);
static_assert(kWholeTiles <= kSumBlocks, "slots");

// A tensor as the tiles see it: rows that follow one another are one row.
struct Flat {
    int64_t rows, cols, stride;
};

int check_tensor(const char* name, int64_t i, const gockpt_grad_tensor& t, Flat* flat) {
    const long long at = static_cast<long long>(i);
    if (!dtype_ok(t.dtype)) return ops_fail(GOCKPT_EINVAL, "%s: tensor %lld: dtype %d", name, at, t.dtype);
    if (t.dst != nullptr && !dtype_ok(t.dst_dtype))
        return ops_fail(GOCKPT_EINVAL, "%s: tensor %lld: dst_dtype %d", name, at, t.dst_dtype);
    if (t.rows < 0 || t.cols < 0 || t.rows > kMaxElems || t.cols > kMaxElems ||
        (t.cols > 0 && t.rows > kMaxElems / t.cols))
        return ops_fail(GOCKPT_EINVAL, "%s: tensor %lld: %lld x %lld elements", name, at,
                        static_cast<long long>(t.rows), static_cast<long long>(t.cols));
    if (t.rows > 1 && (t.stride < t.cols || t.stride > kMaxElems / t.rows))
        return ops_fail(GOCKPT_EINVAL, "%s: tensor %lld: stride %lld for rows of %lld", name, at,
                        static_cast<long long>(t.stride), static_cast<long long>(t.cols));
    *flat = {0, 0, 0};
    if (t.rows == 0 || t.cols == 0) return GOCKPT_OK;
    if (t.data == nullptr || !elem_aligned(t.data, t.dtype))
        return ops_fail(GOCKPT_EINVAL, "%s: tensor %lld: data is null or not aligned to its element", name, at);
    if (t.dst != nullptr && !elem_aligned(t.dst, t.dst_dtype))
        return ops_fail(GOCKPT_EINVAL, "%s: tensor %lld: dst is not aligned to its element", name, at);
    if (t.dst == t.data && (t.dst_dtype != t.dtype || (t.rows > 1 && t.stride != t.cols)))
        return ops_fail(GOCKPT_EINVAL, "%s: tensor %lld: dst is data of another type or layout", name, at);
    *flat = t.rows == 1 || t.stride == t.cols ? Flat{1, t.rows * t.cols, 0} : Flat{t.rows, t.cols, t.stride};
    return GOCKPT_OK;
}

// Calls f(first row, rows, first element of the row, elements) for each tile.
template <class F>
void each_tile(const Flat& x, int dtype, F&& f) {
    const int64_t per_unit = 16 / dtype_bytes(dtype);
    const int64_t units = (x.cols + per_unit - 1) / per_unit;
    if (units <= 0) return;
    if (x.rows == 1 || units * 2 > kTileUnits) {  // pieces of a row
        for (int64_t r = 0; r < x.rows; ++r)
            for (int64_t c = 0; c < x.cols; c += kTileUnits * per_unit)
                f(r, int64_t{1}, c, x.cols - c < kTileUnits * per_unit ? x.cols - c : kTileUnits * per_unit);
    } else {  // several rows
        const int64_t n = kTileUnits / units;
        for (int64_t r = 0; r < x.rows; r += n) f(r, x.rows - r < n ? x.rows - r : n, int64_t{0}, x.cols);
    }
}

int64_t count_tiles(const Flat& x, int dtype) {
    const int64_t per_unit = 16 / dtype_bytes(dtype);
    const int64_t units = (x.cols + per_unit - 1) / per_unit;
    if (units <= 0) return 0;
    if (x.rows == 1 || units * 2 > kTileUnits) return x.rows * ((units + kTileUnits - 1) / kTileUnits);
    const int64_t n = kTileUnits / units;
    return (x.rows + n - 1) / n;
}

int count_list(const char* name, const gockpt_grad_tensor* tensors, int64_t count, int64_t* ntiles) {
    *ntiles = 0;
    if (count < 0 || (count > 0 && tensors == nullptr)) return ops_fail(GOCKPT_EINVAL, "%s: tensor list", name);
    for (int64_t i = 0; i < count; ++i) {
        Flat x;
        const int rc = check_tensor(name, i, tensors[i], &x);
        if (rc != GOCKPT_OK) return rc;
        *ntiles += count_tiles(x, tensors[i].dtype);
        if (*ntiles >= (int64_t{1} << 24)) return ops_fail(GOCKPT_EINVAL, "%s: too many elements", name);
    }
    return GOCKPT_OK;
}

}  // namespace

}  // namespace gockpt

using namespace gockpt;

struct gockpt_grads {
    uint8_t* ws;
    const GradTile* tiles;
    int ntiles, spins, spins0;
    bool range;                    // a destination has a narrower range than its source
    int64_t src_bytes, dst_bytes;  // of all tensors
};

extern "C" {

int gockpt_grads_bytes(const gockpt_grad_tensor* tensors, int64_t count, size_t* bytes) {
    if (bytes == nullptr) return ops_fail(GOCKPT_EINVAL, "gockpt_grads_bytes: null argument");
    *bytes = 0;
    int64_t ntiles;
    const int rc = count_list("gockpt_grads_bytes", tensors, count, &ntiles);
    if (rc == GOCKPT_OK) *bytes = (kTableOff + ntiles * sizeof(GradTile) + 255) / 256 * 256;
    return rc;
}

int gockpt_grads_create(const gockpt_grad_tensor* tensors, int64_t count, void* workspace, size_t workspace_bytes,
                        void* stream, gockpt_grads** out) {
    const char* name = "gockpt_grads_create";
    if (out == nullptr) return ops_fail(GOCKPT_EINVAL, "%s: null argument", name);
    *out = nullptr;
    int64_t ntiles;
    const int rc = count_list(name, tensors, count, &ntiles);
    if (rc != GOCKPT_OK) return rc;
    if (workspace == nullptr || reinterpret_cast<uintptr_t>(workspace) % 256 != 0)
        return ops_fail(GOCKPT_EINVAL, "%s: the workspace must be 256-byte aligned", name);
    if (workspace_bytes < kTableOff + ntiles * sizeof(GradTile))
        return ops_fail(GOCKPT_ENOMEM, "%s: workspace of %zu bytes", name, workspace_bytes);
    std::vector<uint8_t> head;  // the workspace's contents
    int64_t src_bytes = 0, dst_bytes = 0;
    bool range = false;
    try {
        head.resize(kTableOff + ntiles * sizeof(GradTile));
        for (int i = 0; i < kGroups; ++i)  // the first epoch, 1: cleared slots are not of it
            reinterpret_cast<uint32_t*>(head.data())[i * kGroupWords] = kGroupBlocks;
        GradTile* next = reinterpret_cast<GradTile*>(head.data() + kTableOff);
        for (int64_t i = 0; i < count; ++i) {
            const gockpt_grad_tensor& t = tensors[i];
            Flat x;
            check_tensor(name, i, t, &x);
            const bool in_place = t.dst == nullptr || t.dst == t.data;
            const int dst_dtype = in_place ? t.dtype : t.dst_dtype;
            const int64_t sb = dtype_bytes(t.dtype), db = dtype_bytes(dst_dtype);
            const int64_t dst_cols = in_place ? x.stride : x.cols;
            range |= (dst_dtype == kFP16 && t.dtype != kFP16) || (dst_dtype == kBF16 && t.dtype == kFP32);
            uint8_t* dst = static_cast<uint8_t*>(in_place ? const_cast<void*>(t.data) : t.dst);
            const uint8_t* src = static_cast<const uint8_t*>(t.data);
            each_tile(x, t.dtype, [&](int64_t r, int64_t rows, int64_t c, int64_t cols) {
                GradTile g{};
                g.src = src + (r * x.stride + c) * sb;
                g.dst = dst + (r * dst_cols + c) * db;
                g.stride = x.stride * sb;
                g.dst_row = dst_cols * db;
                g.per_row = static_cast<int32_t>((cols * sb + 15) / 16);
                g.units = static_cast<int32_t>(rows) * g.per_row;
                g.magic = g.per_row > 1 ? static_cast<uint32_t>((uint64_t{1} << 32) / g.per_row) + 1u : 0u;
                g.skip = static_cast<int16_t>(g.per_row * 16 - cols * sb);
                g.dtype = static_cast<int8_t>(t.dtype);
                g.dst_dtype = static_cast<int8_t>(dst_dtype);
                *next++ = g;
                src_bytes += rows * cols * sb;
                dst_bytes += rows * cols * db;
            });
        }
    } catch (...) {
        return ops_fail(GOCKPT_ENOMEM, "%s: out of host memory", name);
    }
    gockpt_grads* list = new (std::nothrow) gockpt_grads;
    if (list == nullptr) return ops_fail(GOCKPT_ENOMEM, "%s: out of host memory", name);
    list->ws = static_cast<uint8_t*>(workspace);
    list->tiles = reinterpret_cast<const GradTile*>(list->ws + kTableOff);
    list->ntiles = static_cast<int>(ntiles);
    const char* again = getenv("GOCKPT_TEST_GRADS_AGAIN");
    list->spins = again != nullptr && again[0] == '1' ? 0 : kWholeSpins;
    list->spins0 = list->spins == 0 ? 0 : kSpins0;
    list->range = range;
    list->src_bytes = src_bytes;
    list->dst_bytes = dst_bytes;
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e = hipMemcpyAsync(workspace, head.data(), head.size(), hipMemcpyHostToDevice, s);
    const hipError_t w = hipStreamSynchronize(s);
    if (e == hipSuccess) e = w;
    if (e != hipSuccess) {
        delete list;
        return ops_fail(GOCKPT_EHIP, "%s: %s", name, hipGetErrorString(e));
    }
    *out = list;
    return GOCKPT_OK;
}

int gockpt_grads_destroy(gockpt_grads* list) {
    delete list;
    return GOCKPT_OK;
}

static int check_norm(const char* name, const void* scale, double max_norm, const void* result) {
    if (result == nullptr || reinterpret_cast<uintptr_t>(result) % 8 != 0)
        return ops_fail(GOCKPT_EINVAL, "%s: the result must be 8-byte aligned device memory", name);
    if (reinterpret_cast<uintptr_t>(scale) % 4 != 0) return ops_fail(GOCKPT_EINVAL, "%s: scale alignment", name);
    if (!(max_norm >= 0.0)) return ops_fail(GOCKPT_EINVAL, "%s: max_norm %g", name, max_norm);
    return GOCKPT_OK;
}

static void launch_scale(const gockpt_grads* list, const gockpt_grad_result* result, hipStream_t s) {
    if (list->ntiles == 0) return;
    const bool nt = list->src_bytes + list->dst_bytes > kCachedScaleBytes;
    hipLaunchKernelGGL(nt ? scale_kernel<true> : scale_kernel<false>, dim3(list->ntiles), dim3(kThreads), 0, s,
                       list->tiles, list->ntiles, result);
}

// The norm, and with clip the scaling.
static int run_list(const char* name, gockpt_grads* list, const float* scale, double max_norm,
                    gockpt_grad_result* result, bool clip, void* stream) {
    if (list == nullptr) return ops_fail(GOCKPT_EINVAL, "%s: null list", name);
    const int rc = check_norm(name, scale, max_norm, result);
    if (rc != GOCKPT_OK) return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int n = list->ntiles;
    uint32_t* sync = reinterpret_cast<uint32_t*>(list->ws);
    uint64_t* slots = reinterpret_cast<uint64_t*>(list->ws + kSlotsOff);
    uint64_t* ranges = reinterpret_cast<uint64_t*>(list->ws + kRangesOff);
    if (n == 0) {
        hipLaunchKernelGGL(result_kernel, dim3(1), dim3(1), 0, s, result, scale, max_norm, true);
    } else if (n <= kWholeTiles) {
        const auto kernel = clip ? list->range ? whole_kernel<true, true> : whole_kernel<true, false>
                                 : list->range ? whole_kernel<false, true> : whole_kernel<false, false>;
        hipLaunchKernelGGL(kernel, dim3(n), dim3(kThreads), 0, s, list->tiles, sync, slots, ranges, list->spins,
                           list->spins0, scale, max_norm, result);
    } else {
        const bool nt = !clip || list->src_bytes > kCachedSumBytes;
        const auto kernel = nt ? list->range ? sumsq_kernel<true, true> : sumsq_kernel<true, false>
                               : list->range ? sumsq_kernel<false, true> : sumsq_kernel<false, false>;
        hipLaunchKernelGGL(kernel, dim3(n < kSumBlocks ? n : kSumBlocks), dim3(kThreads), 0, s, list->tiles, n, sync,
                           slots, ranges, list->spins0, scale, max_norm, result);
        if (clip) launch_scale(list, result, s);
    }
    return ops_launched(name);
}

int gockpt_grads_norm(gockpt_grads* list, const float* scale, double max_norm, gockpt_grad_result* result,
                      void* stream) {
    return run_list("gockpt_grads_norm", list, scale, max_norm, result, false, stream);
}

int gockpt_grads_clip(gockpt_grads* list, const float* scale, double max_norm, gockpt_grad_result* result,
                      void* stream) {
    return run_list("gockpt_grads_clip", list, scale, max_norm, result, true, stream);
}

int gockpt_grads_scale(gockpt_grads* list, const gockpt_grad_result* result, void* stream) {
    const char* name = "gockpt_grads_scale";
    if (list == nullptr) return ops_fail(GOCKPT_EINVAL, "%s: null list", name);
    const int rc = check_norm(name, nullptr, 0.0, result);
    if (rc != GOCKPT_OK) return rc;
    launch_scale(list, result, static_cast<hipStream_t>(stream));
    return ops_launched(name);
}

int gockpt_grads_result(gockpt_grad_result* result, const float* scale, double max_norm, void* stream) {
    const char* name = "gockpt_grads_result";
    const int rc = check_norm(name, scale, max_norm, result);
    if (rc != GOCKPT_OK) return rc;
    hipLaunchKernelGGL(result_kernel, dim3(1), dim3(1), 0, static_cast<hipStream_t>(stream), result, scale, max_norm,
                       false);
    return ops_launched(name);
}

}  // extern "C"
