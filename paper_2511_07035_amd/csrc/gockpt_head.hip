// gockpt_head.hip -- cross entropy of the head's logits over the whole
// vocabulary and its gradients, without keeping the logits.
//
//   l[t][v] = scale <x_t, w_v>,  lse_t = log sum_v exp l[t][v],  loss_t = lse_t - l[t][y_t]
//   z[t][v] = g_t (exp(l[t][v] - lse_t) - [v = y_t]),  dX = scale Z W,  dW = scale Z^T X
//
// Exponentials are taken to the base 2: with l2 = l log2(e), a tile of logits
// leaves each of its tokens the tile's largest l2 and sum of 2^(l2 - largest);
// one wavefront a token joins them.  The gradients compute the logits again in
// pieces of the vocabulary whose Z fits the workspace; a piece's Z is read by two
// products, dW's rows of the piece, which is done, and dX, which is summed in
// fp32 over the pieces.  Tokens that are masked are left out at the start (but by
// the loss of a few): the others are numbered, and every kernel works on so many.
//
// Z is rounded to the inputs' 16-bit type, as the matrix cores take it: each
// term of dX and dW is off by half a step of that type, which the sums average.
// Not so a token's largest term, its target's: what rounding took from that is
// kept, and its product with the target's row of the table is added to dX in fp32
// (root mean square error of dX at 16384 tokens of 2048 columns against float64:
// 0.0029 of its own without, 0.0018 with; its rounding to bf16 alone makes 0.0017),
// and for the first two tokens of each class its product with the hidden row to
// dW, where a class that few tokens have has few terms to average.
// Z is scaled by a power of two, 2^13 / 2^q where 2^q <= max |g| < 2^(q + 1), so
// that fp16 has probabilities down to 2^-37 and nothing overflows; the products
// are scaled back in fp32.  Where each token has a g of its own, fp16 would so keep
// little or nothing of a token whose g is far below the largest (at 2^-20 of it and
// 50304 classes alike a row of dX was off by 5e-4, at 2^-24 by up to 0.7 of itself).
// There dX takes a Z of its own, each token's row lifted by the power of two that
// its g lacks, which a row of dX is divided by again.  dW sums over the tokens and
// keeps the one scale: what fp16 lacks there is 2^-38 of the largest g.  Both
// gradients so take 670 us instead of 600 (2331 x 1160, 32003 classes), as Z is
// stored twice and in pieces half as large; dX alone, whose one Z is the lifted, 381
// instead of 378.
#include "gockpt_mma.h"
#include "gockpt_model_internal.h"

namespace gockpt {

namespace {

constexpr double kLog2e = 1.4426950408889634074;
constexpr float kLn2 = 0.69314718055994530942f;

// ---- the tokens that count --------------------------------------------------------

struct TokenArgs {
    const void* ids;
    int64_t stride, first, low, high, ignore;  // counts: low <= id < high, not ignore
    int32_t tokens, length, rows, wide;
    int32_t reduction;
    int32_t* count;
    int32_t* of_kept;   // token of the k-th that counts
    int32_t* target;    // and its row of the table, -1 where that is another rank's
    // the loss: zeros for masked tokens (null: not wanted)
    float *lse, *logit, *loss;
    // the gradients (null: not)
    const float *lse_in, *grad;
    int32_t* of_token;  // number among those that count, or -1
    int32_t* seen;      // the first of them that have each row of the table, the second (null: not wanted)
    float* base;        // log2(e) lse of the k-th
    float* factor;      // g 2^(13 - q)
    float* up;          // what lifts the k-th's row of Z (null: nothing does)
    float* unscale;     // 2^(q - 13)
};

constexpr int kTokenThreads = 1024, kTokenWaves = kTokenThreads / 64;

__device__ __forceinline__ int64_t target_of(const TokenArgs& a, int32_t t) {
    const int64_t at = a.length == a.stride ? t : static_cast<int64_t>(t / a.length) * a.stride + t % a.length;
    return a.wide ? static_cast<const int64_t*>(a.ids)[at] : static_cast<const int32_t*>(a.ids)[at];
}

__device__ __forceinline__ bool counts(const TokenArgs& a, int64_t id) {
    return id >= a.low && id < a.high && id != a.ignore;
}

// What a lane keeps of a token: its row of the table, or
constexpr int32_t kElsewhere = -1, kMasked = -2;

__device__ __forceinline__ int32_t row_of(const TokenArgs& a, int64_t t) {
    const int64_t id = target_of(a, static_cast<int32_t>(t));
    if (!counts(a, id)) return kMasked;
    const int64_t row = id - a.first;
    return row >= 0 && row < a.rows ? static_cast<int32_t>(row) : kElsewhere;
}

// Up to so many tokens the block that numbers them also fills `seen` (of 2048 in 9
// us); two launches do of more (2331 in 10 us, 16384 in 23; the block alone had to
// store for 20 us and do its atomics for 50).
constexpr int32_t kSeenAlone = 2048;

// A row's entries before any token: rows that no token has keep what the memory
// held, and a reader asks target whether an entry is true.
__device__ __forceinline__ void see_none(const TokenArgs& a, int32_t row) {
    if (a.seen == nullptr || row < 0) return;
    for (int u = 0; u < kSeen; ++u) a.seen[u * static_cast<int64_t>(a.rows) + row] = INT32_MAX;
}

// Token k of its row's: the least number stays in the first entry, and each other
// one, whether it came too late or was there before, goes on to the second, where
// the least of those stays.  That is the same whatever the order.
__device__ __forceinline__ void see(const TokenArgs& a, int32_t k) {
    static_assert(kSeen == 2, "two entries");
    const int32_t row = a.target[k];
    if (row < 0) return;
    const int32_t was = __hip_atomic_fetch_min(a.seen + row, k, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const int32_t other = max(was, k);
    if (other != INT32_MAX)
        __hip_atomic_fetch_min(a.seen + a.rows + row, other, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// g of every token but with GOCKPT_EACH, whose largest magnitude is `most`, and
// what z is scaled by; `all` tokens count.
__device__ __forceinline__ float factor_of_all(const TokenArgs& a, int32_t all, float most, float& up_by) {
    float g = 0.0f;
    if (a.reduction != GOCKPT_EACH) {
        g = a.grad[0];
        if (a.reduction == GOCKPT_MEAN) g = g / static_cast<float>(max(all, 1));
        most = fabsf(g);
    }
    // no power of two makes infinities or NaN finite: they go through
    int q = 0;
    if (most > 0.0f && most <= 3.402823466e38f) q = max(ilogbf(most), -100);
    up_by = ldexpf(1.0f, 13 - q);
    if (threadIdx.x == 0) *a.unscale = ldexpf(1.0f, q - 13);
    return g;
}

// The power of two that lifts a factor of a token to those of the largest g.
__device__ __forceinline__ float up_of(float factor) {
    const float x = fabsf(factor);
    if (!(x > 0.0f && x <= 3.402823466e38f)) return 1.0f;
    return ldexpf(1.0f, min(max(13 - ilogbf(x), 0), 126));
}

// One block: each wavefront counts its stretch of tokens, then numbers it from
// the sum of those before.  A lane holds its first tokens from one pass to the
// other, all 16384 of a block's.
__global__ __launch_bounds__(kTokenThreads) void token_kernel(TokenArgs a) {
    __shared__ int32_t counted[kTokenWaves];
    __shared__ float largest[kTokenWaves];
    constexpr int kHeld = 16;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int32_t each = (a.tokens + kTokenThreads - 1) / kTokenThreads * 64;
    const int64_t from = static_cast<int64_t>(wave) * each;
    const int64_t to = min(from + each, static_cast<int64_t>(a.tokens));
    const bool weighted = a.grad != nullptr && a.reduction == GOCKPT_EACH;
    int32_t held[kHeld];
#pragma unroll
    for (int u = 0; u < kHeld; ++u) {
        const int64_t t = from + 64 * u + lane;
        held[u] = t < to ? row_of(a, t) : kMasked;
    }
    int32_t mine = 0;
    float most = 0.0f;
#pragma unroll
    for (int u = 0; u < kHeld; ++u) {
        mine += held[u] != kMasked;
        if (weighted && held[u] != kMasked) most = fmaxf(most, fabsf(a.grad[from + 64 * u + lane]));
    }
#pragma unroll 4
    for (int64_t t = from + 64 * kHeld + lane; t < to; t += 64) {
        if (row_of(a, t) == kMasked) continue;
        ++mine;
        if (weighted) most = fmaxf(most, fabsf(a.grad[t]));
    }
    for (int d = 32; d > 0; d >>= 1) {
        mine += __shfl_xor(mine, d);
        most = fmaxf(most, __shfl_xor(most, d));
    }
    if (lane == 0) {
        counted[wave] = mine;
        largest[wave] = most;
    }
    __syncthreads();
    int32_t before = 0, all = 0;
    for (int w = 0; w < kTokenWaves; ++w) {
        if (w < wave) before += counted[w];
        all += counted[w];
        most = fmaxf(most, largest[w]);
    }
    float g = 0.0f, up_by = 1.0f;
    if (a.grad != nullptr) {
        g = factor_of_all(a, all, most, up_by);
    } else if (a.unscale != nullptr && threadIdx.x == 0) {
        *a.unscale = 1.0f;  // no tokens: the gradients are sums of nothing, times this
    }
    if (threadIdx.x == 0) *a.count = all;
    const auto number = [&](int64_t t, int32_t row) {
        const bool there = row != kMasked;
        const uint64_t votes = __ballot(there);
        const int32_t k = before + __popcll(votes & ((uint64_t{1} << lane) - 1));
        before += __popcll(votes);
        if (t >= to) return;
        if (there) {
            a.of_kept[k] = static_cast<int32_t>(t);
            a.target[k] = row;
            if (a.tokens <= kSeenAlone) see_none(a, row);
            if (a.grad != nullptr) {
                a.base[k] = a.lse_in[t] * static_cast<float>(kLog2e);
                const float factor = (weighted ? a.grad[t] : g) * up_by;
                a.factor[k] = factor;
                if (a.up != nullptr) a.up[k] = up_of(factor);
            }
        } else {
            if (a.lse != nullptr) a.lse[t] = 0.0f;
            if (a.logit != nullptr) a.logit[t] = 0.0f;
            if (a.loss != nullptr && a.reduction == GOCKPT_EACH) a.loss[t] = 0.0f;
        }
        if (a.of_token != nullptr) a.of_token[t] = there ? k : -1;
    };
#pragma unroll
    for (int u = 0; u < kHeld; ++u)
        if (from + 64 * u < to) number(from + 64 * u + lane, held[u]);
    for (int64_t at = from + 64 * kHeld; at < to; at += 64)
        number(at + lane, at + lane < to ? row_of(a, at + lane) : kMasked);
    if (a.seen == nullptr || a.tokens > kSeenAlone) return;
    __threadfence();
    __syncthreads();
    for (int32_t k = threadIdx.x; k < all; k += kTokenThreads) see(a, k);
}

template <bool kReset>
__global__ __launch_bounds__(256) void seen_kernel(TokenArgs a) {
    const int32_t k = blockIdx.x * 256 + threadIdx.x;
    if (k >= *a.count) return;
    if constexpr (kReset)
        see_none(a, a.target[k]);
    else
        see(a, k);
}

// Up to so many tokens are not numbered, as leaving some out would leave out no
// tile: the k-th is token k, and of those that do not count nothing is used.  That
// is a launch less each way, and one more where dX needs no sums joined (96 tokens
// of 64 columns, 320 classes, both ways: 133 us, numbered 144; one token of 4096
// columns, 32000 classes, its loss: 50.3, numbered 53.7).
constexpr int32_t kFew = 256;

// What the gradients take from token_kernel and of the hidden rows, for so few
// tokens: rows of those that do not count are zeros, as z_kernel makes their z, so
// that they add nothing to dW.  The first block also has the tokens' numbers; count[0] is all of them,
// count[1] as well unless none counts.
__global__ __launch_bounds__(kFew) void few_kernel(TokenArgs a, const uint8_t* hidden, int64_t stride, int32_t cols,
                                                   uint8_t* dst, int64_t dst_stride) {
    const int32_t groups = (cols + 7) / 8;
    for (int32_t at = blockIdx.x * kFew + threadIdx.x; at < groups * a.tokens; at += gridDim.x * kFew) {
        const int32_t t = at / groups, col = (at - t * groups) * 8;
        u32x4 w = {0, 0, 0, 0};
        if (row_of(a, t) != kMasked) w = load8(hidden + t * stride + int64_t{col} * 2, cols - col);
        *reinterpret_cast<u32x4*>(dst + t * dst_stride + col * 2) = w;
    }
    if (blockIdx.x != 0) return;
    __shared__ float largest[kFew / 64];
    const int32_t t = threadIdx.x, row = t < a.tokens ? row_of(a, t) : kMasked;
    const bool there = row != kMasked, weighted = a.reduction == GOCKPT_EACH;
    float most = weighted && there ? fabsf(a.grad[t]) : 0.0f;
    for (int d = 32; d > 0; d >>= 1) most = fmaxf(most, __shfl_xor(most, d));
    if ((t & 63) == 0) largest[t >> 6] = most;
    const int32_t all = __syncthreads_count(there);
    for (int w = 0; w < kFew / 64; ++w) most = fmaxf(most, largest[w]);
    float up_by;
    const float g = factor_of_all(a, all, most, up_by);
    if (t == 0) {
        a.count[0] = a.tokens;
        a.count[1] = all > 0 ? a.tokens : 0;
    }
    if (t < a.tokens) {
        a.target[t] = row;
        a.of_token[t] = there ? t : -1;
        a.base[t] = there ? a.lse_in[t] * static_cast<float>(kLog2e) : 0.0f;
        const float factor = there ? (weighted ? a.grad[t] : g) * up_by : 0.0f;
        a.factor[t] = factor;
        if (a.up != nullptr) a.up[t] = up_of(factor);
        see_none(a, row);
    }
    if (a.seen == nullptr) return;
    __threadfence();
    __syncthreads();
    if (t < a.tokens) see(a, t);
}

// ---- the loss ---------------------------------------------------------------------

struct LossArgs {
    MmaArgs a;       // R: the table, C: the hidden rows that count
    float log2_scale;  // scale log2(e)
    const int32_t* target;
    TokenArgs few;   // with tokens: c is the token itself, whether it counts or not
    float2* part;    // token k's largest l2 and sum in tile r at k * tiles_r + r
    float* logit;    // l2 of its target
};

template <class M>
__device__ __forceinline__ void negate(typename M::Acc& acc) {
#pragma unroll
    for (int i = 0; i < M::kFR; ++i)
#pragma unroll
        for (int j = 0; j < M::kFC; ++j) acc[i][j] = -acc[i][j];
}

template <class M>
__global__ __launch_bounds__(M::kThreads) void logits_kernel(LossArgs g) {
    GOCKPT_MMA_LDS(M)
    const bool few = M::kOneWave || g.few.tokens > 0;
    const int cn = few ? g.few.tokens : *g.a.cn_dev;
    MmaPlace p;
    if (!mma_place(g.a, cn, M::kBR, M::kBC, p)) return;
    int wants[M::kFC];
    if constexpr (M::kOneWave) {  // on their way while the table is read
#pragma unroll
        for (int j = 0; j < M::kFC; ++j) wants[j] = M::c_of(p, j) < cn ? row_of(g.few, M::c_of(p, j)) : kMasked;
    }
    typename M::Acc acc;
    GOCKPT_MMA_RUN(M, g.a, p, cn, g.a.k, acc);
    M::sync();  // the buffers are free
    float2(*waves)[M::kBC] = reinterpret_cast<float2(*)[M::kBC]>(lr0);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    if (g.log2_scale < 0.0f) negate<M>(acc);
    const float scale = fabsf(g.log2_scale);  // >= 0: the largest product with it is the largest logit
    const bool edge = M::first_r(p) + M::kFR * 16 > g.a.rn;
#pragma unroll
    for (int j = 0; j < M::kFC; ++j) {
        const int c = M::c_of(p, j);
        const int want = M::kOneWave ? wants[j] : c >= cn ? kMasked : few ? row_of(g.few, c) : g.target[c];
        // most tiles hold the targets of none of their tokens
        if (__any(want >= M::first_r(p) && want < M::first_r(p) + M::kFR * 16)) {
            float l = 0.0f;
            bool here = false;
#pragma unroll
            for (int i = 0; i < M::kFR; ++i) {
                const int at = want - M::r_of(p, i);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (at == e) {
                        l = acc[i][j][e];
                        here = true;
                    }
            }
            if (here) g.logit[c] = l * scale;
        }
        if (edge) {
#pragma unroll
            for (int i = 0; i < M::kFR; ++i) {
                const int left = g.a.rn - M::r_of(p, i);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (e >= left) acc[i][j][e] = -INFINITY;
            }
        }
        float most = -INFINITY;
#pragma unroll
        for (int i = 0; i < M::kFR; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) most = fmaxf(most, acc[i][j][e]);
        most = fmaxf(most, __shfl_xor(most, 16));
        most = fmaxf(most, __shfl_xor(most, 32));
        // beyond the last row there is nothing, whatever the scale
        most = most == -INFINITY ? most : most * scale;
        // a row of nothing but -inf keeps a sum of 0
        const float from = most == -INFINITY ? 0.0f : most;
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < M::kFR; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                sum += __builtin_amdgcn_exp2f(__builtin_fmaf(acc[i][j][e], scale, -from));
        if (scale == 0.0f && edge) {  // -inf * 0, where each row that is there counts 1
            sum = 0.0f;
#pragma unroll
            for (int i = 0; i < M::kFR; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    sum += acc[i][j][e] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(acc[i][j][e] * scale - from);
        }
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (lane < 16) waves[wave / M::kWC][(wave % M::kWC * M::kFC + j) * 16 + lane] = float2{most, sum};
    }
    M::sync();
    for (int i = threadIdx.x; i < M::kBC; i += M::kThreads) {
        if (p.c0 + i >= cn) break;
        float most = -INFINITY, sum = 0.0f;
#pragma unroll
        for (int w = 0; w < M::kWR; ++w) most = fmaxf(most, waves[w][i].x);
        const float from = most == -INFINITY ? 0.0f : most;
#pragma unroll
        for (int w = 0; w < M::kWR; ++w) sum += waves[w][i].y * __builtin_amdgcn_exp2f(waves[w][i].x - from);
        g.part[static_cast<int64_t>(p.c0 + i) * g.a.tiles_r + p.tile_r] = float2{most, sum};
    }
}

struct JoinArgs {
    const float2* part;
    const int32_t *count, *of_kept, *target;
    TokenArgs few;  // with tokens: the k-th is token k itself, whether it counts or not
    const float* logit2;
    uint32_t tiles_r;
    int32_t reduction;
    float *lse, *logit, *loss;
    float* each;  // the tokens' losses, for their sum
};

// Up to so many tokens one block joins and adds up; 16 lanes take one where it has
// few partials (96 tokens of 3: 5 us, in place of two launches of 4 and 2).
constexpr int kJoinWaves = 16, kJoinAlone = 64, kJoinAloneNarrow = 256;
constexpr uint32_t kJoinFew = 64;

// The sum of all tokens' losses, in an order that is the same on every call.
__device__ __forceinline__ void sum_losses(const JoinArgs& a) {
    __shared__ double sums[kJoinWaves];
    const bool few = a.few.tokens > 0;
    const int32_t count = few ? a.few.tokens : *a.count;
    int32_t kept = count;
    if (few) {
        const int32_t t = threadIdx.x;
        kept = __syncthreads_count(t < count && row_of(a.few, t) != kMasked);
    }
    double total = 0.0;
    for (int32_t k = threadIdx.x; k < count; k += kJoinWaves * 64) total += static_cast<double>(a.each[k]);
    for (int d = 32; d > 0; d >>= 1) total += __shfl_xor(total, d);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = total;
    __syncthreads();
    if (threadIdx.x != 0) return;
    total = 0.0;
    for (int w = 0; w < kJoinWaves; ++w) total += sums[w];
    *a.loss = static_cast<float>(a.reduction == GOCKPT_MEAN ? total / max(kept, 1) : total);
}

// A wavefront a token, or 16 lanes where it has few partials.
template <bool kAlone, int kLanes>
__global__ __launch_bounds__(kAlone ? kJoinWaves * 64 : 256) void join_kernel(JoinArgs a) {
    constexpr int kTokens = (kAlone ? kJoinWaves * 64 : 256) / kLanes;  // of a block at once
    const int lane = threadIdx.x % kLanes;
    const bool few = a.few.tokens > 0;
    const int32_t count = few ? a.few.tokens : *a.count;
    const bool single = a.reduction == GOCKPT_EACH;
    for (int32_t k = blockIdx.x * kTokens + threadIdx.x / kLanes; k < count; k += gridDim.x * kTokens) {
        const float2* p = a.part + static_cast<int64_t>(k) * a.tiles_r;
        const int32_t row = few ? row_of(a.few, k) : a.target[k];
        float most = -INFINITY, sum = 0.0f;
        for (uint32_t i = lane; i < a.tiles_r; i += 4 * kLanes) {
            float2 x[4];  // on their way together
#pragma unroll
            for (int u = 0; u < 4; ++u)
                x[u] = i + kLanes * u < a.tiles_r ? p[i + kLanes * u] : float2{-INFINITY, 0.0f};
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float top = fmaxf(most, x[u].x), from = top == -INFINITY ? 0.0f : top;
                sum = sum * __builtin_amdgcn_exp2f(most - from) + x[u].y * __builtin_amdgcn_exp2f(x[u].x - from);
                most = top;
            }
        }
        float top = most;
        for (int d = kLanes / 2; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
        const float from = top == -INFINITY ? 0.0f : top;
        sum *= __builtin_amdgcn_exp2f(most - from);
        for (int d = kLanes / 2; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
        if (lane == 0) {
            const int32_t t = few ? k : a.of_kept[k];
            const bool there = row != kMasked;
            const float log2_sum = __builtin_amdgcn_logf(sum);
            const float logit2 = row >= 0 ? a.logit2[k] : 0.0f;
            if (a.lse != nullptr) a.lse[t] = there ? (from + log2_sum) * kLn2 : 0.0f;
            if (a.logit != nullptr) a.logit[t] = logit2 * kLn2;
            const float loss = there ? (from - logit2 + log2_sum) * kLn2 : 0.0f;
            if (a.loss != nullptr) {
                if (single)
                    a.loss[t] = loss;
                else
                    a.each[k] = loss;
            }
        }
    }
    if constexpr (kAlone) {
        if (single || a.loss == nullptr) return;
        __threadfence_block();
        __syncthreads();
        sum_losses(a);
    }
}

__global__ __launch_bounds__(kJoinWaves * 64) void sum_kernel(JoinArgs a) { sum_losses(a); }

// ---- the gradients ------------------------------------------------------------------

struct GradArgs {
    MmaArgs a;       // R: the piece's rows of the table, C: the hidden rows that count
    float log2_scale;
    const int32_t* target;
    int32_t first;   // the piece's first row
    const float *base, *factor;
    uint8_t* z;      // token k's row at z + k * z_stride
    int64_t z_stride;
    float* lost;     // what rounding took from the target's z
    // kLifted: the same, each row times up; z null: only these
    const float* up;
    uint8_t* lifted;
    float* lost_lifted;
};

template <class M, bool kLifted>
__global__ __launch_bounds__(M::kThreads) void z_kernel(GradArgs g) {
    GOCKPT_MMA_LDS(M)
    const int cn = *g.a.cn_dev;
    MmaPlace p;
    if (!mma_place(g.a, cn, M::kBR, M::kBC, p)) return;
    typename M::Acc acc;
    GOCKPT_MMA_RUN(M, g.a, p, cn, g.a.k, acc);
    const bool edge = M::first_r(p) + M::kFR * 16 > g.a.rn;
#pragma unroll
    for (int j = 0; j < M::kFC; ++j) {
        const int c = min(M::c_of(p, j), cn - 1);
        const float base = g.base[c], factor = g.factor[c];
        const int row = g.target[c], want = M::c_of(p, j) < cn ? row - g.first : -1;
#pragma unroll
        for (int i = 0; i < M::kFR; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                acc[i][j][e] =
                    __builtin_amdgcn_exp2f(__builtin_fmaf(acc[i][j][e], g.log2_scale, -base)) * factor;
        // most tiles hold the targets of none of their tokens
        if (__any(want >= M::first_r(p) && want < M::first_r(p) + M::kFR * 16)) {
            float z = 0.0f;
            bool here = false;
#pragma unroll
            for (int i = 0; i < M::kFR; ++i) {
                const int at = want - M::r_of(p, i);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (at == e) {
                        z = acc[i][j][e] - factor;
                        acc[i][j][e] = z;
                        here = true;
                    }
            }
            const auto lost_of = [](float x) { return x - elem_to_f32<M::kT>(pack2<M::kT>(x, x) & 0xffff); };
            if (here) g.lost[c] = lost_of(z);
            if (kLifted && here) g.lost_lifted[c] = lost_of(z * g.up[c]);
        }
        // a token that does not count adds nothing, also where its zeros met infinities
        if (__any(row == kMasked)) {
#pragma unroll
            for (int i = 0; i < M::kFR; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][e] = row == kMasked ? 0.0f : acc[i][j][e];
        }
        if (edge) {
#pragma unroll
            for (int i = 0; i < M::kFR; ++i) {
                const int left = g.a.rn - M::r_of(p, i);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (e >= left) acc[i][j][e] = 0.0f;
            }
        }
    }
    M::sync();
    const Store<M> store = GOCKPT_MMA_STORE(M);
    const int wide = (g.a.rn + 7) / 8 * 8;  // the products read whole pieces of 8: zeros behind the last row
    if (!kLifted || g.z != nullptr) {
#pragma unroll
        for (int j = 0; j < M::kFC; ++j)
            store.put(acc, j, g.z, g.z_stride, M::kT, false, 1.0f, M::first_r(p), wide, M::first_c(p, j), cn);
    }
    if constexpr (kLifted) {
#pragma unroll
        for (int j = 0; j < M::kFC; ++j) {
            const float up = g.up[min(M::c_of(p, j), cn - 1)];
#pragma unroll
            for (int i = 0; i < M::kFR; ++i) acc[i][j] *= up;
            store.put(acc, j, g.lifted, g.z_stride, M::kT, false, 1.0f, M::first_r(p), wide, M::first_c(p, j), cn);
        }
    }
}

// ---- host ---------------------------------------------------------------------------

constexpr int64_t kPieceBytes = int64_t{256} << 20;  // of Z: what the last-level cache holds
constexpr int64_t kSliceBytes = int64_t{256} << 20;  // of dX's fp32 sums, where one slice is less

template <int kT>
void start_logits(int shape, const LossArgs& g, hipStream_t s) {
    const dim3 grid(g.a.tiles_r * g.a.tiles_c);
    using W = Mma<kT, kAlongK, kAlongK, 256, 256, 2, 4>;
    using D = Mma<kT, kAlongK, kAlongK, 128, 128, 2, 2>;
    using T = Stream<kT>;
    static_assert(W::kThreads == product_threads(kWide) && D::kThreads == product_threads(kMid) &&
                      T::kThreads == product_threads(kThin),
                  "what too_many_blocks counts");
    if (shape == kWide)
        hipLaunchKernelGGL(logits_kernel<W>, grid, dim3(W::kThreads), 0, s, g);
    else if (shape == kMid)
        hipLaunchKernelGGL(logits_kernel<D>, grid, dim3(D::kThreads), 0, s, g);
    else
        hipLaunchKernelGGL(logits_kernel<T>, grid, dim3(T::kThreads), 0, s, g);
}

template <int kT, bool kLifted>
void start_z(int shape, const GradArgs& g, hipStream_t s) {
    const dim3 grid(g.a.tiles_r * g.a.tiles_c);
    using W = Mma<kT, kAlongK, kAlongK, 256, 256, 2, 4>;
    using D = Mma<kT, kAlongK, kAlongK, 128, 128, 2, 2>;
    using T = Stream<kT>;
    static_assert(W::kThreads == product_threads(kWide) && D::kThreads == product_threads(kMid) &&
                      T::kThreads == product_threads(kThin),
                  "what too_many_blocks counts");
    if (shape == kWide)
        hipLaunchKernelGGL((z_kernel<W, kLifted>), grid, dim3(W::kThreads), 0, s, g);
    else if (shape == kMid)
        hipLaunchKernelGGL((z_kernel<D, kLifted>), grid, dim3(D::kThreads), 0, s, g);
    else
        hipLaunchKernelGGL((z_kernel<T, kLifted>), grid, dim3(T::kThreads), 0, s, g);
}

void place_tiles(MmaArgs& a, const ProductPlan& p) {
    a.tiles_r = p.tiles_r;
    a.tiles_c = p.tiles_c;
    a.splits = 1;
    a.split_k = p.split_k;
}

int check_head(const char* name, const gockpt_head* h, TokenArgs* t) {
    if (h == nullptr) return ops_fail(GOCKPT_EINVAL, "%s: null head", name);
    int rc = check_model_matrix(name, "hidden", &h->hidden, kHalfTypes);
    if (rc == GOCKPT_OK) rc = check_model_matrix(name, "table", &h->table, kHalfTypes);
    if (rc != GOCKPT_OK) return rc;
    if (h->hidden.dtype != h->table.dtype)
        return ops_fail(GOCKPT_EINVAL, "%s: hidden of dtype %d, table of %d", name, h->hidden.dtype, h->table.dtype);
    if (h->hidden.cols != h->table.cols)
        return ops_fail(GOCKPT_EINVAL, "%s: hidden of %lld columns, table of %lld", name,
                        static_cast<long long>(h->hidden.cols), static_cast<long long>(h->table.cols));
    const gockpt_token_ids& y = h->targets;
    if (y.batch < 0 || y.length < 0 || y.batch > kMaxExtent || y.length > kMaxExtent ||
        y.batch * y.length > kMaxExtent)
        return ops_fail(GOCKPT_EINVAL, "%s: %lld x %lld targets", name, static_cast<long long>(y.batch),
                        static_cast<long long>(y.length));
    const int64_t n = y.batch * y.length;
    if (n != h->hidden.rows)
        return ops_fail(GOCKPT_EINVAL, "%s: %lld targets, %lld rows of hidden", name, static_cast<long long>(n),
                        static_cast<long long>(h->hidden.rows));
    if (y.batch > 1 && (y.stride < y.length || y.stride > int64_t{1} << 31))
        return ops_fail(GOCKPT_EINVAL, "%s: targets stride %lld for sequences of %lld", name,
                        static_cast<long long>(y.stride), static_cast<long long>(y.length));
    if (y.bits != 32 && y.bits != 64) return ops_fail(GOCKPT_EINVAL, "%s: targets of %d bits", name, y.bits);
    if (n > 0 && (y.ids == nullptr || reinterpret_cast<uintptr_t>(y.ids) % (y.bits / 8) != 0))
        return ops_fail(GOCKPT_EINVAL, "%s: targets are null or not aligned", name);
    if (h->classes < 0 || (h->classes > 0 && (y.first_id < 0 || y.first_id > h->classes - h->table.rows)))
        return ops_fail(GOCKPT_EINVAL, "%s: rows %lld to %lld of %lld classes", name,
                        static_cast<long long>(y.first_id), static_cast<long long>(y.first_id + h->table.rows),
                        static_cast<long long>(h->classes));
    if (y.first_id > INT64_MAX - kMaxExtent)
        return ops_fail(GOCKPT_EINVAL, "%s: first_id %lld", name, static_cast<long long>(y.first_id));
    if (t != nullptr) {
        t->ids = y.ids;
        t->length = static_cast<int32_t>(y.length);
        t->stride = y.batch > 1 ? y.stride : y.length;
        t->first = y.first_id;
        t->low = h->classes > 0 ? 0 : y.first_id;
        t->high = h->classes > 0 ? h->classes : y.first_id + h->table.rows;
        t->ignore = h->ignore_id;
        t->tokens = static_cast<int32_t>(n);
        t->rows = static_cast<int32_t>(h->table.rows);
        t->wide = y.bits == 64;
    }
    return GOCKPT_OK;
}

int check_blocks(const char* name, const ProductPlan& p) {
    if (too_many_blocks(p))
        return ops_fail(GOCKPT_EINVAL, "%s: a product of %u x %u tiles", name, p.tiles_r, p.tiles_c);
    return GOCKPT_OK;
}

int check_reduction(const char* name, int r) {
    if (r < GOCKPT_EACH || r > GOCKPT_MEAN) return ops_fail(GOCKPT_EINVAL, "%s: reduction %d", name, r);
    return GOCKPT_OK;
}

// Rows that count are taken by their numbers where offsets from the first one
// stay within 32 bits.
bool hidden_in_place(const gockpt_matrix& x) {
    return in_place(x) && (x.rows <= 1 || x.rows * x.stride * 2 < (int64_t{1} << 32));
}

struct LossPlan {
    ProductPlan logits;
    size_t count, of_kept, target, part, logit2, each, hidden, table, bytes;
};

LossPlan plan_loss(const gockpt_head& h) {
    LossPlan p{};
    Parts parts;
    const int64_t n = h.hidden.rows;
    p.logits = plan_product(kAlongAlong, h.table.rows, n, h.table.cols, 1);
    p.count = parts.take(4);
    p.of_kept = parts.take(n * 4);
    p.target = parts.take(n * 4);
    p.part = parts.take(n * p.logits.tiles_r * 8);
    p.logit2 = parts.take(n * 4);
    p.each = parts.take(n * 4);
    p.hidden = parts.take(hidden_in_place(h.hidden) ? 0 : n * copy_stride(h.hidden.cols) * 2);
    p.table = parts.take(copy_bytes(h.table));
    p.bytes = parts.bytes;
    return p;
}

// One piece of the vocabulary: Z, dX and dW of so many rows.
struct Piece {
    ProductPlan z, by_hidden, by_table;
};

struct GradPlan {
    int64_t piece;   // rows of the table in a piece
    Piece full, rest;
    size_t count, unscale, of_kept, target, of_token, seen, base, factor, lost, up, lost_lifted, hidden, table, z, lifted,
        slices_hidden, slices_table, bytes;
    int64_t z_stride;
};

Piece plan_piece(int64_t tokens, int64_t rows, int64_t cols, bool by_hidden, bool by_table, int most_hidden) {
    Piece p{};
    p.z = plan_product(kAlongAlong, rows, tokens, cols, 1);
    if (by_hidden) p.by_hidden = plan_product(kAcrossAlong, cols, tokens, rows, most_hidden);
    if (by_table) p.by_table = plan_product(kAcrossAcross, cols, rows, tokens, 64);
    return p;
}

// Whether dX takes a Z of its own.
bool lifts(const gockpt_head& h, bool by_hidden, int reduction) {
    return by_hidden && h.hidden.dtype == kFP16 && reduction == GOCKPT_EACH;
}

GradPlan plan_grad(const gockpt_head& h, bool by_hidden, bool by_table, bool lifted) {
    GradPlan p{};
    Parts parts;
    const int64_t n = h.hidden.rows, rows = h.table.rows, cols = h.table.cols;
    const int most_hidden = static_cast<int>(
        std::max<int64_t>(1, std::min<int64_t>(64, kSliceBytes / std::max<int64_t>(1, n * cols * 4))));
    const auto cost = [&](int64_t r) {
        const Piece x = plan_piece(n, r, cols, by_hidden, by_table, most_hidden);
        // dX's sums are read and written once a piece
        return x.z.us + x.by_hidden.us + x.by_table.us +
               (by_hidden ? static_cast<double>(n) * static_cast<double>(cols) * 8.0 / 4.5e6 : 0.0);
    };
    const int64_t each = lifted && by_table ? 4 : 2;  // bytes of an element of Z, or of both
    const int64_t most = std::max<int64_t>(256, kPieceBytes / std::max<int64_t>(1, n * each) / 256 * 256);
    p.piece = std::max<int64_t>(rows, 1);
    if (rows > most) {
        // tiles run in rounds: pieces whose tiles fill them, the rest's too
        const int64_t step = std::max<int64_t>(256, most / 32 / 256 * 256);
        double least = -1.0;
        for (int64_t r = most; r >= 256 && r >= most / 2; r -= step) {
            const int64_t whole = rows / r, rest = rows % r;
            const double us = static_cast<double>(whole) * cost(r) + (rest > 0 ? cost(rest) : 0.0);
            if (least < 0.0 || us < least) {
                least = us;
                p.piece = r;
            }
        }
    }
    const int64_t rest = rows % p.piece;
    p.full = plan_piece(n, std::min(p.piece, rows), cols, by_hidden, by_table, most_hidden);
    p.rest = rest > 0 ? plan_piece(n, rest, cols, by_hidden, by_table, p.full.by_hidden.splits) : p.full;
    p.z_stride = up(p.piece, 64) * 2;
    p.count = parts.take(8);
    p.unscale = parts.take(4);
    p.of_kept = parts.take(n * 4);
    p.target = parts.take(n * 4);
    p.of_token = parts.take(n * 4);
    p.base = parts.take(n * 4);
    p.factor = parts.take(n * 4);
    p.lost = parts.take(n * 4);
    if (lifted) {
        p.up = parts.take(n * 4);
        p.lost_lifted = parts.take(n * 4);
    }
    if (by_table) p.seen = parts.take(kSeen * rows * 4);
    p.hidden = parts.take(n * copy_stride(cols) * 2);
    p.table = parts.take(copy_bytes(h.table));
    p.z = parts.take(n * p.z_stride);
    p.lifted = lifted && by_table ? parts.take(n * p.z_stride) : p.z;
    if (by_hidden) p.slices_hidden = parts.take(p.full.by_hidden.splits * n * cols * 4);
    if (by_table) {
        const auto bytes = [&](const ProductPlan& x, int64_t r) { return x.splits > 1 ? x.splits * r * cols * 4 : 0; };
        p.slices_table = parts.take(std::max(bytes(p.full.by_table, std::min(p.piece, rows)), bytes(p.rest.by_table, rest)));
    }
    p.bytes = parts.bytes;
    return p;
}

int check_blocks(const char* name, const GradPlan& p) {
    int rc = GOCKPT_OK;
    for (const ProductPlan& x : {p.full.z, p.full.by_hidden, p.full.by_table, p.rest.z, p.rest.by_hidden, p.rest.by_table})
        if (rc == GOCKPT_OK) rc = check_blocks(name, x);
    return rc;
}

int check_grads(const char* name, const gockpt_head* h, const gockpt_matrix* gx, const gockpt_matrix* gw) {
    if (gx != nullptr) {
        const int rc = check_model_matrix(name, "grad_hidden", gx, kAnyType);
        if (rc != GOCKPT_OK) return rc;
        if (gx->rows != h->hidden.rows || gx->cols != h->hidden.cols)
            return ops_fail(GOCKPT_EINVAL, "%s: grad_hidden of %lld x %lld", name, static_cast<long long>(gx->rows),
                            static_cast<long long>(gx->cols));
    }
    if (gw != nullptr) {
        const int rc = check_model_matrix(name, "grad_table", gw, kAnyType);
        if (rc != GOCKPT_OK) return rc;
        if (gw->rows != h->table.rows || gw->cols != h->table.cols)
            return ops_fail(GOCKPT_EINVAL, "%s: grad_table of %lld x %lld", name, static_cast<long long>(gw->rows),
                            static_cast<long long>(gw->cols));
    }
    return GOCKPT_OK;
}

}  // namespace

}  // namespace gockpt

using namespace gockpt;

extern "C" {

int gockpt_head_loss_bytes(const gockpt_head* head, size_t* bytes) {
    const char* name = "gockpt_head_loss_bytes";
    if (bytes == nullptr) return ops_fail(GOCKPT_EINVAL, "%s: null argument", name);
    *bytes = 0;
    int rc = check_head(name, head, nullptr);
    if (rc != GOCKPT_OK) return rc;
    const LossPlan p = plan_loss(*head);
    rc = check_blocks(name, p.logits);
    if (rc == GOCKPT_OK) *bytes = p.bytes;
    return rc;
}

int gockpt_head_loss(const gockpt_head* head, int reduction, float* loss, float* lse, float* logit, void* workspace,
                     size_t workspace_bytes, void* stream) {
    const char* name = "gockpt_head_loss";
    TokenArgs t{};
    int rc = check_head(name, head, &t);
    if (rc == GOCKPT_OK) rc = check_reduction(name, reduction);
    if (rc == GOCKPT_OK && loss != nullptr && head->classes > 0)
        rc = ops_fail(GOCKPT_EINVAL, "%s: the loss of a range of the classes", name);
    for (const float* p : {loss, lse, logit})
        if (rc == GOCKPT_OK && reinterpret_cast<uintptr_t>(p) % 4 != 0)
            rc = ops_fail(GOCKPT_EINVAL, "%s: an output is not aligned", name);
    if (rc != GOCKPT_OK) return rc;
    const LossPlan p = plan_loss(*head);
    rc = check_blocks(name, p.logits);
    if (rc == GOCKPT_OK) rc = check_workspace(name, workspace, workspace_bytes, p.bytes);
    if (rc != GOCKPT_OK) return rc;
    if (loss == nullptr && lse == nullptr && logit == nullptr) return GOCKPT_OK;
    if (t.tokens == 0 && (loss == nullptr || reduction == GOCKPT_EACH)) return GOCKPT_OK;
    hipStream_t s = static_cast<hipStream_t>(stream);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    t.reduction = reduction;
    t.count = reinterpret_cast<int32_t*>(ws + p.count);
    t.of_kept = reinterpret_cast<int32_t*>(ws + p.of_kept);
    t.target = reinterpret_cast<int32_t*>(ws + p.target);
    t.lse = lse;
    t.logit = logit;
    t.loss = loss;
    LossArgs g{};
    JoinArgs j{};
    const bool few = t.tokens <= kFew && p.logits.tiles_r > 0 && p.logits.tiles_c > 0;
    if (few)
        g.few = j.few = t;
    else
        hipLaunchKernelGGL(token_kernel, dim3(1), dim3(kTokenThreads), 0, s, t);
    Copies copies;
    const Source table = copies.source_of(head->table, ws + p.table);
    g.a.r = table.data;
    g.a.r_stride = table.stride;
    if (hidden_in_place(head->hidden)) {
        g.a.c = static_cast<const uint8_t*>(head->hidden.data);
        g.a.c_stride = (head->hidden.rows > 1 ? head->hidden.stride : head->hidden.cols) * 2;
        g.a.c_rows = few ? nullptr : t.of_kept;
    } else {
        const Source hidden = copies.rows_of(head->hidden, few ? nullptr : t.of_kept, few ? nullptr : t.count,
                                             head->hidden.rows, ws + p.hidden);
        g.a.c = hidden.data;
        g.a.c_stride = hidden.stride;
    }
    copies.launch(s);
    g.a.rn = t.rows;
    g.a.cn = t.tokens;
    g.a.cn_dev = t.count;
    g.a.k = static_cast<int32_t>(head->table.cols);
    place_tiles(g.a, p.logits);
    g.log2_scale = static_cast<float>(static_cast<double>(head->scale) * kLog2e);
    g.target = t.target;
    g.part = reinterpret_cast<float2*>(ws + p.part);
    g.logit = reinterpret_cast<float*>(ws + p.logit2);
    if (g.a.tiles_r > 0 && g.a.tiles_c > 0) {
        if (head->table.dtype == kBF16)
            start_logits<kBF16>(p.logits.shape, g, s);
        else
            start_logits<kFP16>(p.logits.shape, g, s);
    }
    j.part = g.part;
    j.count = t.count;
    j.of_kept = t.of_kept;
    j.target = t.target;
    j.logit2 = g.logit;
    j.tiles_r = g.a.tiles_r;
    j.reduction = reduction;
    j.lse = lse;
    j.logit = logit;
    j.loss = loss;
    j.each = reinterpret_cast<float*>(ws + p.each);
    const bool narrow = g.a.tiles_r <= kJoinFew;
    if (t.tokens <= (narrow ? kJoinAloneNarrow : kJoinAlone)) {
        hipLaunchKernelGGL((narrow ? join_kernel<true, 16> : join_kernel<true, 64>), dim3(1), dim3(kJoinWaves * 64), 0, s, j);
    } else {
        const int tokens = narrow ? 16 : 4;
        hipLaunchKernelGGL((narrow ? join_kernel<false, 16> : join_kernel<false, 64>),
                           dim3(std::min((t.tokens + tokens - 1) / tokens, kUnits * 8)), dim3(256), 0, s, j);
        if (loss != nullptr && reduction != GOCKPT_EACH)
            hipLaunchKernelGGL(sum_kernel, dim3(1), dim3(kJoinWaves * 64), 0, s, j);
    }
    return ops_launched(name);
}

int gockpt_head_grad_bytes(const gockpt_head* head, const gockpt_matrix* grad_hidden,
                           const gockpt_matrix* grad_table, size_t* bytes) {
    const char* name = "gockpt_head_grad_bytes";
    if (bytes == nullptr) return ops_fail(GOCKPT_EINVAL, "%s: null argument", name);
    *bytes = 0;
    int rc = check_head(name, head, nullptr);
    if (rc == GOCKPT_OK) rc = check_grads(name, head, grad_hidden, grad_table);
    if (rc != GOCKPT_OK) return rc;
    // of any reduction
    const bool by_hidden = grad_hidden != nullptr, by_table = grad_table != nullptr;
    const bool lifted = lifts(*head, by_hidden, GOCKPT_EACH);
    const GradPlan p = plan_grad(*head, by_hidden, by_table, lifted);
    rc = check_blocks(name, p);
    size_t most = p.bytes;
    if (rc == GOCKPT_OK && lifted && p.piece < head->table.rows) {  // in one piece there is more with a Z for dX
        const GradPlan q = plan_grad(*head, by_hidden, by_table, false);
        rc = check_blocks(name, q);
        most = std::max(most, q.bytes);
    }
    if (rc == GOCKPT_OK) *bytes = most;
    return rc;
}

int gockpt_head_grad(const gockpt_head* head, const float* lse, int reduction, const float* grad,
                     const gockpt_matrix* grad_hidden, const gockpt_matrix* grad_table, int accumulate,
                     void* workspace, size_t workspace_bytes, void* stream) {
    const char* name = "gockpt_head_grad";
    TokenArgs t{};
    int rc = check_head(name, head, &t);
    if (rc == GOCKPT_OK) rc = check_grads(name, head, grad_hidden, grad_table);
    if (rc == GOCKPT_OK) rc = check_reduction(name, reduction);
    if (rc == GOCKPT_OK && t.tokens > 0 && (lse == nullptr || grad == nullptr))
        rc = ops_fail(GOCKPT_EINVAL, "%s: null lse or grad", name);
    for (const float* p : {lse, grad})
        if (rc == GOCKPT_OK && reinterpret_cast<uintptr_t>(p) % 4 != 0)
            rc = ops_fail(GOCKPT_EINVAL, "%s: lse or grad is not aligned", name);
    if (rc != GOCKPT_OK) return rc;
    const bool lifted = lifts(*head, grad_hidden != nullptr, reduction);
    const GradPlan p = plan_grad(*head, grad_hidden != nullptr, grad_table != nullptr, lifted);
    rc = check_blocks(name, p);
    if (rc == GOCKPT_OK) rc = check_workspace(name, workspace, workspace_bytes, p.bytes);
    if (rc != GOCKPT_OK) return rc;
    const int64_t rows = head->table.rows, cols = head->table.cols;
    const bool by_hidden = grad_hidden != nullptr && t.tokens > 0 && cols > 0;
    const bool by_table = grad_table != nullptr && rows > 0 && cols > 0 && !(accumulate && t.tokens == 0);
    if (!by_hidden && !by_table) return GOCKPT_OK;
    hipStream_t s = static_cast<hipStream_t>(stream);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    t.reduction = reduction;
    t.count = reinterpret_cast<int32_t*>(ws + p.count);
    t.of_kept = reinterpret_cast<int32_t*>(ws + p.of_kept);
    t.target = reinterpret_cast<int32_t*>(ws + p.target);
    t.of_token = reinterpret_cast<int32_t*>(ws + p.of_token);
    t.lse_in = lse;
    t.grad = t.tokens > 0 ? grad : nullptr;
    if (by_table) t.seen = reinterpret_cast<int32_t*>(ws + p.seen);
    t.base = reinterpret_cast<float*>(ws + p.base);
    t.factor = reinterpret_cast<float*>(ws + p.factor);
    if (lifted) t.up = reinterpret_cast<float*>(ws + p.up);
    float* const lost = reinterpret_cast<float*>(ws + p.lost);
    // what dX is made of
    float* const lost_hidden = lifted ? reinterpret_cast<float*>(ws + p.lost_lifted) : lost;
    uint8_t* const z_hidden = ws + (lifted ? p.lifted : p.z);
    t.unscale = reinterpret_cast<float*>(ws + p.unscale);
    const int64_t hidden_stride = copy_stride(cols) * 2;
    const bool few = t.tokens > 0 && t.tokens <= kFew;
    // dX goes where it belongs at once: c is the token, and there is one sum
    const bool direct = few && by_hidden && rows > 0 && p.piece >= rows && p.full.by_hidden.splits == 1 &&
                        p.full.by_hidden.shape != kWide;
    Copies copies;
    const Source table = copies.source_of(head->table, ws + p.table);
    if (few) {
        const int64_t pieces = (cols + 7) / 8 * t.tokens;
        hipLaunchKernelGGL(few_kernel, dim3(std::min<int64_t>((pieces + kFew - 1) / kFew, kUnits * 8)), dim3(kFew), 0, s,
                           t, static_cast<const uint8_t*>(head->hidden.data), head->hidden.stride * 2,
                           static_cast<int32_t>(cols), ws + p.hidden, hidden_stride);
    } else {
        hipLaunchKernelGGL(token_kernel, dim3(1), dim3(kTokenThreads), 0, s, t);
        if (t.seen != nullptr && t.tokens > kSeenAlone) {
            const dim3 grid((t.tokens + 255) / 256);
            hipLaunchKernelGGL(seen_kernel<true>, grid, dim3(256), 0, s, t);
            hipLaunchKernelGGL(seen_kernel<false>, grid, dim3(256), 0, s, t);
        }
        copies.rows_of(head->hidden, t.of_kept, t.count, t.tokens, ws + p.hidden);
    }
    copies.launch(s);
    const int dtype = head->table.dtype;
    float* slices = reinterpret_cast<float*>(ws + p.slices_hidden);
    for (int64_t first = 0; first < rows; first += p.piece) {
        const int64_t here = std::min(p.piece, rows - first);
        const Piece& plan = here == p.piece ? p.full : p.rest;
        if (t.tokens > 0) {
            GradArgs g{};
            g.a.r = table.data + first * table.stride;
            g.a.r_stride = table.stride;
            g.a.c = ws + p.hidden;
            g.a.c_stride = hidden_stride;
            g.a.rn = static_cast<int32_t>(here);
            g.a.cn = t.tokens;
            g.a.cn_dev = t.count;
            g.a.k = static_cast<int32_t>(cols);
            place_tiles(g.a, plan.z);
            g.log2_scale = static_cast<float>(static_cast<double>(head->scale) * kLog2e);
            g.target = t.target;
            g.first = static_cast<int32_t>(first);
            g.base = t.base;
            g.factor = t.factor;
            g.z = lifted && !by_table ? nullptr : ws + p.z;
            g.z_stride = p.z_stride;
            g.lost = lost;
            g.up = t.up;
            g.lifted = z_hidden;
            g.lost_lifted = lost_hidden;
            if (dtype == kBF16)
                start_z<kBF16, false>(plan.z.shape, g, s);
            else if (lifted)
                start_z<kFP16, true>(plan.z.shape, g, s);
            else
                start_z<kFP16, false>(plan.z.shape, g, s);
        }
        if (by_hidden) {
            MmaArgs a{};
            a.r = table.data + first * table.stride;
            a.r_stride = table.stride;
            a.c = z_hidden;
            a.c_stride = p.z_stride;
            a.rn = static_cast<int32_t>(cols);
            a.cn = t.tokens;
            a.cn_dev = t.count;
            a.k = static_cast<int32_t>(here);
            StoreArgs o{};
            if (direct) {
                o.out = static_cast<uint8_t*>(const_cast<void*>(grad_hidden->data));
                o.stride = (t.tokens > 1 ? grad_hidden->stride : cols) * dtype_bytes(grad_hidden->dtype);
                o.dtype = grad_hidden->dtype;
                o.alpha = head->scale;
                o.beta = t.unscale;
                o.owner = t.target;
                o.fix = lost_hidden;
                o.up = t.up;
            } else {
                o.slices = slices;
                o.add = first > 0;
            }
            launch_product(kAcrossAlong, dtype, plan.by_hidden, a, o, s);
        }
        if (by_table) {
            MmaArgs a{};
            a.r = ws + p.hidden;
            a.r_stride = hidden_stride;
            a.c = ws + p.z;
            a.c_stride = p.z_stride;
            a.rn = static_cast<int32_t>(cols);
            a.cn = static_cast<int32_t>(here);
            a.k = t.tokens;
            a.k_dev = few ? t.count + 1 : t.count;
            const int64_t stride = (rows > 1 ? grad_table->stride : cols) * dtype_bytes(grad_table->dtype);
            FinishArgs f{};
            f.out = static_cast<uint8_t*>(const_cast<void*>(grad_table->data)) + first * stride;
            f.stride = stride;
            f.dtype = grad_table->dtype;
            f.accumulate = accumulate != 0;
            f.alpha = head->scale;
            f.beta = t.unscale;
            StoreArgs o{};
            o.seen = t.seen;
            o.seen_step = rows;
            o.owner = t.target;
            o.fix = lost;
            o.first = static_cast<int32_t>(first);
            if (plan.by_table.splits > 1) {
                o.slices = reinterpret_cast<float*>(ws + p.slices_table);
                launch_product(kAcrossAcross, dtype, plan.by_table, a, o, s);
                f.slices = o.slices;
                f.slice_step = here * cols;
                f.count = plan.by_table.splits;
                f.rows = static_cast<int32_t>(here);
                f.cols = static_cast<int32_t>(cols);
                launch_finish(f, s);
            } else {
                o.out = f.out;
                o.stride = f.stride;
                o.dtype = f.dtype;
                o.accumulate = f.accumulate;
                o.alpha = f.alpha;
                o.beta = f.beta;
                launch_product(kAcrossAcross, dtype, plan.by_table, a, o, s);
            }
        }
    }
    if (by_hidden && !direct) {
        FinishArgs f{};
        f.slices = slices;
        f.slice_step = int64_t{t.tokens} * cols;
        f.count = rows > 0 ? p.full.by_hidden.splits : 0;
        f.rows = t.tokens;
        f.cols = static_cast<int32_t>(cols);
        f.of_row = t.of_token;
        f.out = static_cast<uint8_t*>(const_cast<void*>(grad_hidden->data));
        f.stride = (t.tokens > 1 ? grad_hidden->stride : cols) * dtype_bytes(grad_hidden->dtype);
        f.dtype = grad_hidden->dtype;
        f.alpha = head->scale;
        f.beta = t.unscale;
        f.up = t.up;
        f.fix = lost_hidden;
        f.fix_row = t.target;
        f.fix_from = table.data;
        f.fix_stride = table.stride;
        f.fix_dtype = dtype;
        launch_finish(f, s);
    }
    return ops_launched(name);
}

}  // extern "C"
