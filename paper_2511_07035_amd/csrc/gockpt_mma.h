// gockpt_mma.h -- the matrix product that the head's loss and the 8-bit linear
// layers share, on gfx950's matrix cores.
//
//   out[c][r] = sum over k of R(r, k) * C(c, k)
//
// R's index r runs along the output's rows (its contiguous direction), C's
// index c counts them.  Each operand is 16 bits wide and lies either with k
// contiguous (kAlongK: element (i, k) at data + i * stride + k) or with i
// contiguous (kAcrossK: at data + k * stride + i).
//
// One block computes a tile of kBR x kBC over steps of 64 k.  Tiles go from
// global memory straight into LDS, 16 bytes a lane, into one of two buffers
// while the other is multiplied.  The copy writes lanes one after another, so
// the order that keeps LDS reads free of bank conflicts is made by permuting
// which 16 bytes a lane fetches, and undone by the reads:
//   kAlongK   rows of 128 bytes, 16-byte piece p of row i at p ^ (i / 2 & 7); a
//             fragment is one 16-byte read a lane, 16 lanes at a time, and of 16
//             rows every other one lies in the same banks (with i & 7 the counters
//             showed as many cycles of conflicts as of reads).
//   kAcrossK  rows of k, 32-byte unit u of row k at u ^ f(k), f = 0, 3, 5, 6 for k &
//             3, and the lowest bit of that turned where k & 8: the eight rows that
//             32 lanes of a transposing read take then lie in different banks.
// A fragment of step s + 1 is read while step s is multiplied, across the
// barrier between two tiles as well: a wave holds the last step's fragments
// in registers when it passes it.
//
// Over many tiles of k blocks begin at different ones, and take the rest in turn:
// blocks that march through k together wait for the same few channels of the
// caches, which hold one k of all rows.  us, all from the first k and in turn (r x c
// x k): both along k, 8192 x 8192 x 8192 766 and 746, 16384 x 4096 x 5120 511 and 492;
// R across, 2048 x 16384 x 8192 405 and 385.  With fewer tiles, and where no operand
// lies along k, blocks in step share more of the L2: 8192 x 16384 x 2048 404 and 415,
// 4096 x 16384 x 4096 (R across) 388 and 397, 2048 x 8192 x 16384 (both) 374 and 379.
// (Products one at a time, 20 ms apart.  One after another the card's clock falls,
// and the long ones take 2 to 20% more, those in turn no less than the others.)
#pragma once

#include "gockpt_ops_internal.h"

namespace gockpt {

typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef f32x4 f32x4_any __attribute__((aligned(2)));

enum Lay : int { kAlongK = 0, kAcrossK = 1 };

constexpr int kStepK = 64;  // k of one LDS tile
constexpr int kTurns = 32;        // tiles of k that blocks begin at,
constexpr int kTurnsFrom = 64;    // with more of them than this

#define GOCKPT_LDS __attribute__((address_space(3)))

// What every product is given.  Strides are in bytes.
struct MmaArgs {
    const uint8_t* r;
    const uint8_t* c;
    int64_t r_stride, c_stride;
    int32_t rn, cn;          // extents of r and c
    int32_t k;               // of k; a multiple of 8 for kAlongK
    const int32_t* cn_dev;   // the extent of c, or of k, on the device (null: as above);
    const int32_t* k_dev;    // at most what the field above says
    const int32_t* c_rows;   // kAlongK: row of C that stands at c (null: c itself)
    uint32_t tiles_r, tiles_c;
    int32_t splits, split_k;  // slices of k and their length, a multiple of 64
};

// 16 r by 16 c by 32 k.  (32 by 32 by 16 needs as many cycles and registers, and
// was slower: 8192 x 8192 x 8192 817 us against 744.)
template <int kT>
__device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c) {
    if constexpr (kT == kBF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c,
                                                       0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0,
                                                      0, 0);
}

__device__ __forceinline__ int unit_swizzle(int k) { return (((k & 3) << 1) | ((k ^ (k >> 1)) & 1)) ^ (k >> 3 & 1); }

template <class T>
__device__ __forceinline__ T* uniform(T* p) {
    const uint64_t v = reinterpret_cast<uint64_t>(p);
    const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v));
    const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v >> 32));
    return reinterpret_cast<T*>(static_cast<uint64_t>(hi) << 32 | lo);
}

// threadIdx.x, of which the compiler does not know that it is what it was before a
// product: what comes after it computes its addresses then, and the product does
// not go without their registers.
__device__ __forceinline__ int this_thread() {
    int t = threadIdx.x;
    asm volatile("" : "+v"(t));
    return t;
}

// This wave's copies into LDS have landed (vmcnt 0; the builtin tells the
// compiler too, which else waits again before reads).
__device__ __forceinline__ void wait_copies() { __builtin_amdgcn_s_waitcnt(0x0f70); }

// The tile of one operand: kB indexes by 64 k, filled by kWaves wavefronts.
template <int kLay, int kB, int kWaves>
struct Filler {
    static constexpr int kPieces = kB / 8 / kWaves;  // copies of 1 KiB a wave makes for a tile
    static constexpr int kRowLanes = kB / 8;         // kAcrossK: lanes that copy a row of k
    static_assert(kPieces >= 1, "each wave copies");

    // kAcrossK: a wave's copies lie 16 rows of k apart, at the same piece each
    static_assert(kLay == kAlongK || 64 / kRowLanes * kWaves == 16, "rows of k alike in the swizzle");
    static constexpr int kOffs = kLay == kAlongK ? kPieces : 1;

    const uint8_t* base;  // of the tile's first index, at k = 0
    int64_t step;         // bytes from one tile of k to the next
    uint32_t apart;       // kAcrossK: from one copy to the next
    uint32_t off[kOffs];
    uint32_t back[kOffs];  // from off to a place that is there in every tile of k
    int k_of[kOffs];       // first k of the lane's piece within the tile

    // Tile at index i0 < n of the operand; rows: see MmaArgs.c_rows.
    __device__ __forceinline__ void init(const uint8_t* data, int64_t stride, int i0, int n, const int32_t* rows,
                                         int lane, int wave) {
        if constexpr (kLay == kAlongK) {
            base = uniform(rows != nullptr ? data : data + static_cast<int64_t>(i0) * stride);
            step = 2 * kStepK;
#pragma unroll
            for (int j = 0; j < kPieces; ++j) {
                const int piece = (lane & 7) ^ (((j * kWaves + wave) & 1) * 4 + (lane >> 4));
                const int i = min((j * kWaves + wave) * 8 + (lane >> 3), n - 1 - i0);
                const uint32_t row = rows != nullptr ? static_cast<uint32_t>(rows[i0 + i]) : static_cast<uint32_t>(i);
                off[j] = row * static_cast<uint32_t>(stride) + piece * 16;
                back[j] = piece * 16;
                k_of[j] = piece * 8;
            }
        } else {
            base = uniform(data + static_cast<int64_t>(i0) * 2);
            step = stride * kStepK;
            apart = 16 * static_cast<uint32_t>(stride);
            const int k = wave * (64 / kRowLanes) + lane / kRowLanes, at = lane % kRowLanes;
            int piece = ((at >> 1) ^ (unit_swizzle(k) & (kRowLanes / 2 - 1))) * 2 + (at & 1);
            if (i0 + piece * 8 >= n) piece = 0;
            back[0] = static_cast<uint32_t>(k) * static_cast<uint32_t>(stride);
            off[0] = back[0] + piece * 16;
            k_of[0] = k;
        }
    }

    // Starts the copies of the tile of k that begins at tile * 64.  kWhole: all
    // its k are there; else `left` are.
    template <bool kWhole>
    __device__ __forceinline__ void fill(GOCKPT_LDS uint8_t* lds, int tile, int left, int wave) {
#if defined(__HIP_DEVICE_COMPILE__)  // the host's pass does not know the buffer's type
        __amdgpu_buffer_rsrc_t res = __builtin_amdgcn_make_buffer_rsrc(
            const_cast<uint8_t*>(base + static_cast<int64_t>(tile) * step), 0, 0xffffffff, 0x00027000);
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            GOCKPT_LDS void* const to = (GOCKPT_LDS void*)(lds + (j * kWaves + wave) * 1024);
            if constexpr (kLay == kAlongK) {
                const uint32_t at = kWhole || k_of[j] < left ? off[j] : off[j] - back[j];
                __builtin_amdgcn_raw_ptr_buffer_load_lds(res, to, 16, at, 0, 0, 0);
            } else if constexpr (kWhole) {
                __builtin_amdgcn_raw_ptr_buffer_load_lds(res, to, 16, off[0], j * apart, 0, 0);
            } else {  // in place of a row that is not there, the tile's first
                const uint32_t at = k_of[0] + j * 16 < left ? off[0] + j * apart : off[0] - back[0];
                __builtin_amdgcn_raw_ptr_buffer_load_lds(res, to, 16, at, 0, 0, 0);
            }
        }
#endif
    }

    // Zeros in place of what the wave copied beyond the last k, once landed.
    __device__ __forceinline__ void clear(GOCKPT_LDS uint8_t* lds, int left, int lane, int wave) {
#pragma unroll
        for (int j = 0; j < kPieces; ++j)
            if ((kLay == kAlongK ? k_of[j % kOffs] : k_of[0] + j * 16) >= left)
                *reinterpret_cast<GOCKPT_LDS u32x4*>(lds + (j * kWaves + wave) * 1024 + lane * 16) = u32x4{0, 0, 0, 0};
    }

};

// Fragments of 16 indexes by 32 k: lane l holds index l & 15, k 8 * (l >> 4) on.
template <int kLay, int kB, int kBlocks>
struct Reader {
    uint32_t at[kLay == kAlongK ? 2 : kBlocks];  // of each step's piece, or of each block of indexes

    __device__ __forceinline__ void init(int first, int lane) {
        const int t = lane & 15, up = lane >> 4;
        if constexpr (kLay == kAlongK) {
#pragma unroll
            for (int s = 0; s < 2; ++s) at[s] = (first + t) * 128 + (((4 * s + up) ^ (lane >> 1 & 7)) << 4);
        } else {
            const int k = up * 8 + (t >> 2), f = unit_swizzle(k) & (kB / 16 - 1);
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) at[b] = k * (2 * kB) + ((first / 16 + b) ^ f) * 32 + (t & 3) * 8;
        }
    }

    // Block b (16 indexes from first on), step s of the tile's two.
    __device__ __forceinline__ u32x4 read(const GOCKPT_LDS uint8_t* lds, int b, int s) const {
        if constexpr (kLay == kAlongK) {
            return *reinterpret_cast<const GOCKPT_LDS u32x4*>(lds + at[s] + b * 16 * 128);
        } else {
            GOCKPT_LDS s16x4* p = (GOCKPT_LDS s16x4*)(lds + at[b] + s * 32 * (2 * kB));
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(p);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(p + 4 * (2 * kB) / 8);
            const u32x2 a = __builtin_bit_cast(u32x2, lo), c = __builtin_bit_cast(u32x2, hi);
            return u32x4{a.x, a.y, c.x, c.y};
        }
    }
};

// Tile of r0.. x c0.. that a block computes, and its slice of k.
struct MmaPlace {
    int r0, c0, split;
    uint32_t tile_r;
};

// Blocks go to the 8 XCDs in turn; each XCD takes one run of tiles, in groups
// of 4 tiles of c (2, 8 and 16 were slower by up to 4%), so that the blocks that
// run on it together read few different tiles and find the others' in its L2.
// Only the tiles below cn are shared out: were the others' blocks to end at
// once, the last XCDs' would, and the others work as long as ever.
__device__ __forceinline__ bool mma_place(const MmaArgs& a, int cn, int br, int bc, MmaPlace& p) {
    const uint32_t tiles_c = static_cast<uint32_t>((cn + bc - 1) / bc);
    const uint32_t n = a.tiles_r * tiles_c, all = n * a.splits;
    uint32_t id = blockIdx.x;
    if (id >= all) return false;
    const uint32_t each = all / 8, over = all % 8, xcd = id % 8, at = id / 8;
    id = xcd * each + min(xcd, over) + at;
    const uint32_t split = id / n;
    id -= split * n;
    const uint32_t group = id / (4 * a.tiles_r), first = group * 4;
    const uint32_t wide = min(tiles_c - first, 4u);
    id -= group * 4 * a.tiles_r;
    p.tile_r = id / wide;
    p.r0 = static_cast<int>(p.tile_r) * br;
    p.c0 = static_cast<int>(first + id % wide) * bc;
    p.split = static_cast<int>(split);
    return true;
}

template <int kT_, int kRLay, int kCLay, int kBR_, int kBC_, int kWR_, int kWC_>
struct Mma {
    static constexpr int kT = kT_, kBR = kBR_, kBC = kBC_, kWR = kWR_, kWC = kWC_;
    static constexpr bool kBothAcross = kRLay == kAcrossK && kCLay == kAcrossK;
    // whether StoreArgs' corrections are made; C along k, the widest tiles have no registers for it
    static constexpr bool kFixes = kBothAcross || (kRLay == kAcrossK && kBR < 256);
    static constexpr int kWaves = kWR * kWC, kThreads = kWaves * 64;
    static constexpr int kFR = kBR / kWR / 16, kFC = kBC / kWC / 16;  // fragments of a wave
    static constexpr int kRBytes = kBR * kStepK * 2, kCBytes = kBC * kStepK * 2;
    static constexpr bool kOneWave = false;
    static_assert(kFR % 2 == 0 && kFC >= 1, "fragments of a wave");

    using Acc = f32x4[kFR][kFC];

    struct State {
        Filler<kRLay, kBR, kWaves> fr;
        Filler<kCLay, kBC, kWaves> fc;
        Reader<kRLay, kBR, kFR> rr;
        Reader<kCLay, kBC, kFC> rc;
        int lane, wave, k;
        int from, whole;  // the k tile to begin with, of so many whole ones
    };

    // Which tile of k comes as the tile-th: the whole ones in turn from st.from on.
    template <bool kWhole>
    static __device__ __forceinline__ int turned(const State& st, int tile) {
        if (kWhole || tile < st.whole) {
            tile += st.from;
            tile -= tile >= st.whole ? st.whole : 0;
        }
        return tile;
    }

    template <bool kWhole>
    static __device__ __forceinline__ void fill(State& st, GOCKPT_LDS uint8_t* r, GOCKPT_LDS uint8_t* c, int tile) {
        const int left = st.k - tile * kStepK;
        tile = turned<kWhole>(st, tile);
        st.fr.template fill<kWhole>(r, tile, left, st.wave);
        st.fc.template fill<kWhole>(c, tile, left, st.wave);
    }

    // The tile's copies have landed for all waves; nobody reads the other buffer any more.
    template <bool kWhole>
    static __device__ __forceinline__ void land(State& st, GOCKPT_LDS uint8_t* r, GOCKPT_LDS uint8_t* c, int tile) {
        wait_copies();
        const int left = st.k - tile * kStepK;
        if (!kWhole && left < kStepK) {
            st.fr.clear(r, left, st.lane, st.wave);
            st.fc.clear(c, left, st.lane, st.wave);
        }
        __syncthreads();
    }

    // A step's fragments of C, and one half of R's.
    struct Cols {
        u32x4 f[kFC];
    };
    struct Half {
        u32x4 f[kFR / 2];
    };

    static __device__ __forceinline__ void read(const State& st, Cols& x, const GOCKPT_LDS uint8_t* c, int s) {
#pragma unroll
        for (int j = 0; j < kFC; ++j) x.f[j] = st.rc.read(c, j, s);
    }

    static __device__ __forceinline__ void read(const State& st, Half& x, const GOCKPT_LDS uint8_t* r, int s, int h) {
#pragma unroll
        for (int i = 0; i < kFR / 2; ++i) x.f[i] = st.rr.read(r, h * (kFR / 2) + i, s);
    }

    static __device__ __forceinline__ void multiply(const Half& r, const Cols& c, int h, Acc& acc) {
#pragma unroll
        for (int i = 0; i < kFR / 2; ++i)
#pragma unroll
            for (int j = 0; j < kFC; ++j)
                acc[h * (kFR / 2) + i][j] = mma<kT>(r.f[i], c.f[j], acc[h * (kFR / 2) + i][j]);
    }

    // Asks for an even mix of half a step's products with the reads for the next
    // half (and, in a tile's last one, the copies): left alone, the compiler puts
    // each read right before its use.
    static constexpr int kHalfReads = kFR / 2 * (kRLay == kAlongK ? 1 : 2);
    static constexpr int kColReads = kFC * (kCLay == kAlongK ? 1 : 2);
    static constexpr int kCopies = (kBR + kBC) / 8 / kWaves;
    template <int kReads, int kCopied>
    static __device__ __forceinline__ void mix() {
        constexpr int kProducts = kFR / 2 * kFC;
        int reads = 0, copies = 0;
#pragma unroll
        for (int i = 0; i < kProducts; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
#pragma unroll
            for (; reads * kProducts < (i + 1) * kReads; ++reads) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
#pragma unroll
            for (; copies * kProducts < (i + 1) * kCopied; ++copies) __builtin_amdgcn_sched_group_barrier(0x20, 1, 0);
        }
    }

    // One tile of k: reads the rest of `r`, `c`, starts reading the next ones.
    // kInner: the next two tiles are there in full.
    template <bool kInner>
    static __device__ __forceinline__ void tile(State& st, Half& r0, Cols& c0, Acc& acc, GOCKPT_LDS uint8_t* r,
                                                GOCKPT_LDS uint8_t* c, GOCKPT_LDS uint8_t* nr, GOCKPT_LDS uint8_t* nc,
                                                int t, int tiles) {
        Half r1;
        Cols c1;
        read(st, r1, r, 0, 1);
        multiply(r0, c0, 0, acc);
        mix<kHalfReads, 0>();
        read(st, r0, r, 1, 0);
        read(st, c1, c, 1);
        multiply(r1, c0, 1, acc);
        mix<kHalfReads + kColReads, 0>();
        read(st, r1, r, 1, 1);
        multiply(r0, c1, 0, acc);
        mix<kHalfReads, 0>();
        if (kInner || t + 1 < tiles) {
            land<kInner>(st, nr, nc, t + 1);
            read(st, r0, nr, 0, 0);
            read(st, c0, nc, 0);
            if (kInner || t + 2 < tiles) fill<kInner>(st, r, c, t + 2);
        }
        multiply(r1, c1, 1, acc);
        if (kInner) mix<kHalfReads + kColReads, kCopies>();
    }

    // acc = the block's tile of the product over its slice of k.  The LDS
    // buffers are separate objects so that the compiler knows a copy into one
    // from a read of the other.
    static __device__ __forceinline__ void run(const MmaArgs& a, const MmaPlace& p, int cn, int k_all,
                                               GOCKPT_LDS uint8_t* r0, GOCKPT_LDS uint8_t* c0,
                                               GOCKPT_LDS uint8_t* r1, GOCKPT_LDS uint8_t* c1, Acc& acc) {
#pragma unroll
        for (int i = 0; i < kFR; ++i)
#pragma unroll
            for (int j = 0; j < kFC; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        State st;
        const int thread = threadIdx.x;
        st.lane = thread & 63;
        st.wave = __builtin_amdgcn_readfirstlane(thread >> 6);
        const int64_t k0 = static_cast<int64_t>(p.split) * a.split_k;
        st.k = static_cast<int>(min(static_cast<int64_t>(a.split_k), k_all - k0));
        if (st.k <= 0) return;
        const int tiles = (st.k + kStepK - 1) / kStepK;
        st.fr.init(a.r + k0 * (kRLay == kAlongK ? 2 : a.r_stride), a.r_stride, p.r0, a.rn, nullptr, st.lane, st.wave);
        st.fc.init(a.c + k0 * (kCLay == kAlongK ? 2 : a.c_stride), a.c_stride, p.c0, cn,
                   kCLay == kAlongK ? a.c_rows : nullptr, st.lane, st.wave);
        st.rr.init(st.wave / kWC * (kFR * 16), st.lane);
        st.rc.init(st.wave % kWC * (kFC * 16), st.lane);
        st.whole = st.k / kStepK;
        st.from = kCLay == kAlongK && st.whole > kTurnsFrom ? (p.r0 / kBR + p.c0 / kBC) % kTurns : 0;
        fill<false>(st, r0, c0, 0);
        land<false>(st, r0, c0, 0);
        Half fr;
        Cols fc;
        read(st, fr, r0, 0, 0);
        read(st, fc, c0, 0);
        if (tiles > 1) fill<false>(st, r1, c1, 1);
        int t = 0;
        for (; t + 3 < st.whole; t += 2) {
            tile<true>(st, fr, fc, acc, r0, c0, r1, c1, t, tiles);
            tile<true>(st, fr, fc, acc, r1, c1, r0, c0, t + 1, tiles);
        }
        for (; t < tiles; t += 2) {
            tile<false>(st, fr, fc, acc, r0, c0, r1, c1, t, tiles);
            if (t + 1 < tiles) tile<false>(st, fr, fc, acc, r1, c1, r0, c0, t + 1, tiles);
        }
    }

    // All wavefronts are through with the product.
    static __device__ __forceinline__ void sync() { __syncthreads(); }

    // Where the wavefront's fragments begin.
    static __device__ __forceinline__ int first_r(const MmaPlace& p) {
        return p.r0 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / kWC * kFR * 16;
    }
    static __device__ __forceinline__ int first_c(const MmaPlace& p, int j) {
        return p.c0 + (__builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % kWC * kFC + j) * 16;
    }
    // The r of this lane's four elements of fragments (i, ..), from the first on,
    // and the c of those of fragments (.., j).
    static __device__ __forceinline__ int r_of(const MmaPlace& p, int i) {
        return first_r(p) + i * 16 + 4 * ((this_thread() & 63) >> 4);
    }
    static __device__ __forceinline__ int c_of(const MmaPlace& p, int j) { return first_c(p, j) + (this_thread() & 15); }
};

// The product of at most 32 c, both operands along k: R is read once, and that is
// the time it takes.  A block takes 32 r, each of its wavefronts every fourth tile
// of k: R's through buffers of its own, kAhead of them on their way, C's straight
// into registers, with no barrier before the sums of the four are put together.
// 32000 x 1 x 4096, 262 MB not read before: 46 us; R's fragments loaded into
// registers, whose every load takes a quarter of 32 lines, 53; tiles of 128 r, of
// which a compute unit has one with 16 KiB on their way, 58.
template <int kT_>
struct Stream {
    static constexpr int kT = kT_, kBR = 32, kBC = 32, kWR = 1, kWC = 1, kFR = 2, kFC = 2;
    static constexpr int kWaves = 4, kThreads = 256, kAhead = 4;
    static constexpr int kTile = 32 * kStepK * 2;
    static constexpr int kRBytes = kWaves * kTile, kCBytes = kWaves * kTile;
    static constexpr bool kOneWave = true;  // the first wavefront has the sum
    static constexpr bool kFixes = false;
    using Acc = f32x4[2][2];

    struct State {
        Filler<kAlongK, 32, 1> fill;
        Reader<kAlongK, 32, 2> reader;
        const uint8_t* c[2];  // this lane's index of each block of C at the first k, its quarter's piece
        int lane, wave, k, from, whole;

        // The wavefront's t-th tile of k: the whole ones in turn, from another one
        // in each block (49 us from the first one in all).
        __device__ __forceinline__ int turned(int t) const {
            if (t < whole) {
                t += from;
                t -= t >= whole ? whole : 0;
            }
            return t * kWaves + wave;
        }

        template <bool kWhole>
        __device__ __forceinline__ void load(GOCKPT_LDS uint8_t* r, u32x4 (&f)[4], int t) {
            const int tile = turned(t), left = k - tile * kStepK;
            fill.template fill<kWhole>(r, tile, left, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) {  // step i / 2, block i % 2
                const uint8_t* p = c[i % 2] + static_cast<int64_t>(tile) * (2 * kStepK);
                const bool there = kWhole || (4 * (i / 2) + (lane >> 4)) * 8 < left;
                // the tile's first piece is there
                const u32x4 x = *reinterpret_cast<const u32x4*>(there ? p + i / 2 * 64 : p - (lane >> 4) * 16);
                f[i] = there ? x : u32x4{0, 0, 0, 0};
            }
        }

        template <bool kWhole>
        __device__ __forceinline__ void multiply(GOCKPT_LDS uint8_t* r, const u32x4 (&f)[4], int t, Acc& acc) {
            if (!kWhole) {
                const int left = k - turned(t) * kStepK;
                wait_copies();
                if (left < kStepK) fill.clear(r, left, lane, 0);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {  // step i / 2, block i % 2 of r
                const u32x4 x = reader.read(r, i % 2, i / 2);
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[i % 2][j] = mma<kT>(x, f[i / 2 * 2 + j], acc[i % 2][j]);
            }
        }
    };

    static __device__ __forceinline__ void run(const MmaArgs& a, const MmaPlace& p, int cn, int k_all,
                                               GOCKPT_LDS uint8_t* b0, GOCKPT_LDS uint8_t* b1, GOCKPT_LDS uint8_t* b2,
                                               GOCKPT_LDS uint8_t* b3, Acc& acc) {
        acc[0][0] = acc[0][1] = acc[1][0] = acc[1][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        State st;
        st.lane = threadIdx.x & 63;
        st.wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int64_t k0 = static_cast<int64_t>(p.split) * a.split_k;
        st.k = static_cast<int>(min(static_cast<int64_t>(a.split_k), k_all - k0));
        GOCKPT_LDS uint8_t* const first = b0;
        b0 += st.wave * kTile;
        b1 += st.wave * kTile;
        b2 += st.wave * kTile;
        b3 += st.wave * kTile;
        if (st.k > 0) {
            st.fill.init(a.r + k0 * 2, a.r_stride, p.r0, a.rn, nullptr, st.lane, 0);
            st.reader.init(0, st.lane);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int at = min(p.c0 + j * 16 + (st.lane & 15), cn - 1);
                st.c[j] = a.c + k0 * 2 + (a.c_rows != nullptr ? a.c_rows[at] : at) * a.c_stride + (st.lane >> 4) * 16;
            }
            const int tiles = ((st.k + kStepK - 1) / kStepK - st.wave + kWaves - 1) / kWaves;  // wave, wave + 4, ...
            st.whole = (st.k / kStepK - st.wave + kWaves - 1) / kWaves;
            st.from = st.whole > 0 ? static_cast<int>(p.tile_r % st.whole) : 0;
            u32x4 f[kAhead][4];
            int t = 0;
            const auto next = [&](GOCKPT_LDS uint8_t* b, u32x4 (&g)[4], int u) {
                st.template multiply<true>(b, g, u, acc);
                st.template load<true>(b, g, u + kAhead);
                // else the compiler waits once for all four tiles
                __builtin_amdgcn_sched_barrier(0);
            };
            if (2 * kAhead <= st.whole) {
                // the loop's loads in the loop's order: waits then count them
                st.template load<true>(b0, f[0], 0);
                __builtin_amdgcn_sched_barrier(0);
                st.template load<true>(b1, f[1], 1);
                __builtin_amdgcn_sched_barrier(0);
                st.template load<true>(b2, f[2], 2);
                __builtin_amdgcn_sched_barrier(0);
                st.template load<true>(b3, f[3], 3);
                __builtin_amdgcn_sched_barrier(0);
                do {
                    next(b0, f[0], t);
                    next(b1, f[1], t + 1);
                    next(b2, f[2], t + 2);
                    next(b3, f[3], t + 3);
                    t += kAhead;
                } while (t + 2 * kAhead <= st.whole);
            } else {
                if (0 < tiles) st.template load<false>(b0, f[0], 0);
                if (1 < tiles) st.template load<false>(b1, f[1], 1);
                if (2 < tiles) st.template load<false>(b2, f[2], 2);
                if (3 < tiles) st.template load<false>(b3, f[3], 3);
            }
            const auto last = [&](GOCKPT_LDS uint8_t* b, u32x4 (&g)[4], int u) {
                if (u < tiles) {
                    st.template multiply<false>(b, g, u, acc);
                    if (u + kAhead < tiles) st.template load<false>(b, g, u + kAhead);
                }
            };
            for (; t < tiles; t += kAhead) {
                last(b0, f[0], t);
                last(b1, f[1], t + 1);
                last(b2, f[2], t + 2);
                last(b3, f[3], t + 3);
            }
        }
        if (st.wave > 0) {
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<GOCKPT_LDS f32x4*>(b0 + (q * 64 + st.lane) * 16) = acc[q / 2][q % 2];
        }
        __syncthreads();
        if (st.wave > 0) return;
#pragma unroll
        for (int w = 1; w < kWaves; ++w) {
#pragma unroll
            for (int q = 0; q < 4; ++q)
                acc[q / 2][q % 2] +=
                    *reinterpret_cast<const GOCKPT_LDS f32x4*>(first + w * kTile + (q * 64 + st.lane) * 16);
        }
    }

    // One wavefront is left.
    static __device__ __forceinline__ void sync() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }
    static __device__ __forceinline__ int first_r(const MmaPlace& p) { return p.r0; }
    static __device__ __forceinline__ int first_c(const MmaPlace& p, int j) { return p.c0 + j * 16; }
    static __device__ __forceinline__ int r_of(const MmaPlace& p, int i) {
        return p.r0 + i * 16 + 4 * ((threadIdx.x & 63) >> 4);
    }
    static __device__ __forceinline__ int c_of(const MmaPlace& p, int j) { return p.c0 + j * 16 + (threadIdx.x & 15); }
};

// Where a product's values go.
struct StoreArgs {
    uint8_t* out;       // row c at out + c * stride bytes
    int64_t stride;
    int32_t dtype, accumulate;
    float alpha;        // factor of every value,
    const float* beta;  // and one on the device (null: 1)
    float* slices;      // not null: fp32 sums instead, slice s at s * cn * rn, unscaled;
    int32_t add;        // added to what is there
    // Corrections of single terms; R lies across k.  C too, and `seen` not null: fix[k]
    // R(r, k) is added to c's sum, for the k that `seen` names for c (entry u of c at
    // seen[u * seen_step + first + c], kSeen of them) and whose owner[k] is first + c;
    // other entries may hold anything.  C along k, `owner` not null and the tile not
    // kWide: fix[c] R(r, k) is, with k = owner[c]; of -1 nothing is added, below that
    // the sum is 0.
    const int32_t* seen;
    int64_t seen_step;
    const int32_t* owner;
    const float* fix;
    int32_t first;
    const float* up;  // with these, C along k: c's sum is up[c] times too large, a power of two (null: none is)
};
constexpr int kSeen = 2;

// In steps over all of a lane's terms, as each step waits for memory: one term after
// another took 13 us a tile.
template <class M>
__device__ __forceinline__ void add_fixes(const MmaArgs& a, const StoreArgs& o, const MmaPlace& p, int cn, int k_all,
                                          typename M::Acc& acc) {
    constexpr int kTerms = M::kBothAcross ? kSeen : 1;
    int k[M::kFC][kTerms];
    float x[M::kFC][kTerms];
#pragma unroll
    for (int j = 0; j < M::kFC; ++j) {
        const int c = min(M::c_of(p, j), cn - 1);
#pragma unroll
        for (int u = 0; u < kTerms; ++u)
            k[j][u] = M::kBothAcross ? o.seen[u * o.seen_step + o.first + c] : o.owner[c];
    }
#pragma unroll
    for (int j = 0; j < M::kFC; ++j) {
        const int c = min(M::c_of(p, j), cn - 1);
#pragma unroll
        for (int u = 0; u < kTerms; ++u) {
            const bool there = static_cast<uint32_t>(k[j][u]) < static_cast<uint32_t>(k_all);
            const int of = there ? k[j][u] : 0;
            x[j][u] = o.fix[M::kBothAcross ? of : c];
            if (M::kBothAcross ? o.owner[of] != o.first + c || !there : k[j][u] == -1) k[j][u] = -1;
        }
    }
#pragma unroll
    for (int j = 0; j < M::kFC; ++j) {
        bool some = false;
#pragma unroll
        for (int u = 0; u < kTerms; ++u) some = some || k[j][u] != -1;
        if (!__any(some)) continue;
        u32x2 w[kTerms][M::kFR];
#pragma unroll
        for (int u = 0; u < kTerms; ++u)
#pragma unroll
            for (int i = 0; i < M::kFR; ++i) {
                const int r = M::r_of(p, i);
                w[u][i] = u32x2{0, 0};
                if (k[j][u] >= 0 && r < a.rn)
                    w[u][i] = *reinterpret_cast<const u32x2*>(a.r + k[j][u] * a.r_stride + r * 2);
            }
#pragma unroll
        for (int u = 0; u < kTerms; ++u)
#pragma unroll
            for (int i = 0; i < M::kFR; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float add = x[j][u] * elem_to_f32<M::kT>(w[u][i][e / 2] >> (16 * (e & 1)) & 0xffff);
                    // x of what is not there may be anything
                    acc[i][j][e] = k[j][u] < -1 ? 0.0f : k[j][u] >= 0 ? acc[i][j][e] + add : acc[i][j][e];
                }
    }
    if constexpr (!M::kBothAcross) {
        if (o.up == nullptr) return;
#pragma unroll
        for (int j = 0; j < M::kFC; ++j) {
            const float down = 1.0f / o.up[min(M::c_of(p, j), cn - 1)];
#pragma unroll
            for (int i = 0; i < M::kFR; ++i) acc[i][j] *= down;
        }
    }
}

template <int kT>
__device__ __forceinline__ u32x2 pack4(f32x4 x) {
    return u32x2{pack2<kT>(x[0], x[1]), pack2<kT>(x[2], x[3])};
}

// n <= 8 values of 16 bits that are there at p, from w; with accumulate
// round(old + x) for the fp32 values x.
template <int kT>
__device__ __forceinline__ void add8(uint8_t* p, const float (&x)[8], int n) {
    uint16_t* q = reinterpret_cast<uint16_t*>(p);
    if (n >= 8) {
        u32x4 w = *reinterpret_cast<const u32x4_any*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] = pack2<kT>(elem_to_f32<kT>(w[i] & 0xffff) + x[2 * i], elem_to_f32<kT>(w[i] >> 16) + x[2 * i + 1]);
        *reinterpret_cast<u32x4_any*>(p) = w;
    } else {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < n) q[i] = static_cast<uint16_t>(pack2<kT>(elem_to_f32<kT>(q[i]) + x[i], 0.0f));
    }
}

// The n > 0 values of 16 bits at p, of which 8 are taken; zeros behind them.
__device__ __forceinline__ u32x4 load8(const uint8_t* p, int n) {
    u32x4 w = {0, 0, 0, 0};
    if (n >= 8) {
        w = *reinterpret_cast<const u32x4_any*>(p);
    } else {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < n) w[i / 2] |= static_cast<uint32_t>(reinterpret_cast<const uint16_t*>(p)[i]) << (16 * (i & 1));
    }
    return w;
}

// Four values along r.  x is rounded once; with accumulate the sum is.
__device__ __forceinline__ void store4(uint8_t* p, int dtype, bool accumulate, f32x4 x, int n) {
    if (dtype == kFP32) {
        if (n >= 4) {
            f32x4_any* q = reinterpret_cast<f32x4_any*>(p);
            *q = accumulate ? *q + x : x;
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (i < n) {
                    float* q = reinterpret_cast<float*>(p) + i;
                    *q = accumulate ? *q + x[i] : x[i];
                }
        }
        return;
    }
    if (accumulate) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) {
                const uint16_t old = reinterpret_cast<const uint16_t*>(p)[i];
                x[i] += dtype == kBF16 ? elem_to_f32<kBF16>(old) : elem_to_f32<kFP16>(old);
            }
    }
    const u32x2 w = dtype == kBF16 ? pack4<kBF16>(x) : pack4<kFP16>(x);
    if (n >= 4) {
        *reinterpret_cast<u32x2_any*>(p) = w;
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < n) reinterpret_cast<uint16_t*>(p)[i] = static_cast<uint16_t>(w[i / 2] >> (16 * (i & 1)));
    }
}

// A block's tile to memory.  A lane holds four values along r of each of its
// columns c, and stores of those would touch 16 rows at 32 bytes each (268 MB of
// bf16 took 78 us more than no stores at all, and take 46 so).  So each wavefront
// turns 16 columns at a time in LDS that it alone uses by then, and stores whole
// stretches of a row, 16 bytes a lane.  The 16-byte piece p of column c lies at p ^
// c: writes and reads of 16 lanes meet every bank once.
template <class M>
struct Store {
    static constexpr int kPieces = M::kFR * 4;    // of 4 values of 32 bits, of a column of the wavefront's tile
    static constexpr int kHalves = M::kFR * 2;    // of 8 values of 16 bits
    static constexpr int kBytes = 16 * kPieces * 16;  // a wavefront's

    GOCKPT_LDS uint8_t* lds;

    // The wavefront's part of the tile buffers; all are free.
    __device__ __forceinline__ Store(GOCKPT_LDS uint8_t* r0, GOCKPT_LDS uint8_t* c0, GOCKPT_LDS uint8_t* r1,
                                     GOCKPT_LDS uint8_t* c1) {
        constexpr int kInR = M::kRBytes / kBytes, kInC = M::kCBytes / kBytes;
        static_assert(2 * (kInR + kInC) >= M::kWaves, "room for each wavefront");
        int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        GOCKPT_LDS uint8_t* at = r0;
        if (w >= kInR) {
            w -= kInR;
            at = r1;
            if (w >= kInR) {
                w -= kInR;
                at = c0;
                if (w >= kInC) {
                    w -= kInC;
                    at = c1;
                }
            }
        }
        lds = at + w * kBytes;
    }

    // Columns c0 to c0 + 15 (those below cn) of fragments acc[..][j], first r r0,
    // `rn` r in all; row c at out + c * stride.
    __device__ __forceinline__ void put(const typename M::Acc& acc, int j, uint8_t* out, int64_t stride, int dtype,
                                        bool accumulate, float alpha, int r0, int rn, int c0, int cn) const {
        const int lane = this_thread() & 63, c = lane & 15, up = lane >> 4;
        if (dtype == kFP32 || accumulate) {
#pragma unroll
            for (int i = 0; i < M::kFR; ++i)
                *reinterpret_cast<GOCKPT_LDS f32x4*>(
                    lds + (c * kPieces + ((i * 4 + up) ^ (c & (kPieces - 1)))) * 16) = acc[i][j] * alpha;
            wave_sync();
            if (dtype == kFP32) {
#pragma unroll 4
                for (int s = 0; s < kPieces / 4; ++s) {
                    const int at = s * 64 + lane, row = at / kPieces, piece = at % kPieces, n = rn - r0 - piece * 4;
                    const f32x4 x = *reinterpret_cast<const GOCKPT_LDS f32x4*>(
                        lds + (row * kPieces + (piece ^ (row & (kPieces - 1)))) * 16);
                    if (c0 + row < cn && n > 0)
                        store4(out + (c0 + row) * stride + static_cast<int64_t>(r0 + piece * 4) * 4, kFP32, accumulate,
                               x, n);
                }
            } else {
#pragma unroll 2
                for (int s = 0; s < kHalves / 4; ++s) {
                    const int at = s * 64 + lane, row = at / kHalves, piece = at % kHalves, n = rn - r0 - piece * 8;
                    float x[8];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const f32x4 y = *reinterpret_cast<const GOCKPT_LDS f32x4*>(
                            lds + (row * kPieces + ((piece * 2 + h) ^ (row & (kPieces - 1)))) * 16);
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[4 * h + e] = y[e];
                    }
                    if (c0 + row < cn && n > 0) {
                        uint8_t* p = out + (c0 + row) * stride + static_cast<int64_t>(r0 + piece * 8) * 2;
                        if (dtype == kBF16)
                            add8<kBF16>(p, x, n);
                        else
                            add8<kFP16>(p, x, n);
                    }
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < M::kFR; ++i) {
                const f32x4 x = acc[i][j] * alpha;
                const u32x2 w = dtype == kBF16 ? pack4<kBF16>(x) : pack4<kFP16>(x);
                *reinterpret_cast<GOCKPT_LDS u32x2*>(
                    lds + (c * kHalves + ((i * 2 + up / 2) ^ (c & (kHalves - 1)))) * 16 + up % 2 * 8) = w;
            }
            wave_sync();
#pragma unroll 4
            for (int s = 0; s < kHalves / 4; ++s) {
                const int at = s * 64 + lane, row = at / kHalves, piece = at % kHalves, n = rn - r0 - piece * 8;
                const u32x4 w = *reinterpret_cast<const GOCKPT_LDS u32x4*>(
                    lds + (row * kHalves + (piece ^ (row & (kHalves - 1)))) * 16);
                if (c0 + row >= cn || n <= 0) continue;
                uint8_t* p = out + (c0 + row) * stride + static_cast<int64_t>(r0 + piece * 8) * 2;
                if (n >= 8) {
                    *reinterpret_cast<u32x4_any*>(p) = w;
                } else {
#pragma unroll
                    for (int e = 0; e < 7; ++e)
                        if (e < n) reinterpret_cast<uint16_t*>(p)[e] = static_cast<uint16_t>(w[e / 2] >> (16 * (e & 1)));
                }
            }
        }
        wave_sync();
    }

    // LDS operations of one wavefront are carried out in order: only the
    // compiler has to keep them so.
    static __device__ __forceinline__ void wave_sync() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }
};

template <class M>
__device__ __forceinline__ void store_tile(const Store<M>& store, const MmaArgs& a, const StoreArgs& o,
                                           const MmaPlace& p, int cn, const typename M::Acc& acc) {
    uint8_t* out = o.out;
    int64_t stride = o.stride;
    int dtype = o.dtype;
    bool accumulate = o.accumulate != 0;
    float alpha = o.alpha * (o.beta != nullptr ? *o.beta : 1.0f);
    if (o.slices != nullptr) {
        out = reinterpret_cast<uint8_t*>(o.slices + static_cast<int64_t>(p.split) * a.cn * a.rn);
        stride = static_cast<int64_t>(a.rn) * 4;
        dtype = kFP32;
        accumulate = o.add != 0;
        alpha = 1.0f;
    }
#pragma unroll
    for (int j = 0; j < M::kFC; ++j)
        store.put(acc, j, out, stride, dtype, accumulate, alpha, M::first_r(p), a.rn, M::first_c(p, j), cn);
}

#define GOCKPT_MMA_LDS(M)                                              \
    __shared__ __attribute__((aligned(1024))) uint8_t lr0[M::kRBytes]; \
    __shared__ __attribute__((aligned(1024))) uint8_t lc0[M::kCBytes]; \
    __shared__ __attribute__((aligned(1024))) uint8_t lr1[M::kRBytes]; \
    __shared__ __attribute__((aligned(1024))) uint8_t lc1[M::kCBytes];

#define GOCKPT_MMA_RUN(M, a, p, cn, k, acc)                                                     \
    M::run(a, p, cn, k, (GOCKPT_LDS uint8_t*)lr0, (GOCKPT_LDS uint8_t*)lc0,                     \
           (GOCKPT_LDS uint8_t*)lr1, (GOCKPT_LDS uint8_t*)lc1, acc);                            \
    if (M::kOneWave && threadIdx.x >= 64) return

// Once all wavefronts are through with the product.
#define GOCKPT_MMA_STORE(M)                                                                       \
    Store<M>((GOCKPT_LDS uint8_t*)lr0, (GOCKPT_LDS uint8_t*)lc0, (GOCKPT_LDS uint8_t*)lr1, \
             (GOCKPT_LDS uint8_t*)lc1)

}  // namespace gockpt
