// The head's kernels and their launches: softmax cross entropy over a vocabulary without its logits, and its gradient.  The losses of
// a single target (cgx_head.hip) and of a teacher's entries (cgx_distill.hip) share them: what differs is a template parameter, Softmax.
//
// With x the hidden states of the N tokens that count, W the weight, z = x W^T:
//   loss call      z tile by tile; each tile leaves its rows' largest logit and sum of exp(z - largest), which a last kernel joins
//   gradient call  for each piece of the vocabulary: z again, d = dloss (exp(z - lse) - [v = target]) into the workspace,
//                  dx += d W, dW = d^T x
// 2 N V H operations for the loss, 2 N V H + 4 N V H for the gradient, against (N + V) H elements read: above some hundred
// tokens everything is bound by the matrix cores, below by reading W.
#pragma once

#include "cgx_head.h"

#include "cgx_head_gemm.h"

namespace cgx {
namespace {

using namespace gemm;

constexpr float kLog2e = 1.44269504088896340736f;

struct Header {
    int32_t count;           // tokens that count
    float unscale;           // what the products of d are multiplied by
};

// What the softmax is taken of: the logits, with one target a row; or the logits over a temperature, where a row has a teacher's entries
// instead (which cgx_distill.hip takes care of, but for the logits that a call's tiles pick out for it).
struct Targets {
    static constexpr bool kTargets = true;
    struct Picks {};
    static __device__ __forceinline__ float of(float z) { return z; }
};

// The entries of a row, sorted by id: where those of each 64 columns of the vocabulary begin (10 bits) and how many they are (6 bits; 63: or
// more).  A wave's tile is 64 columns wide, so a lane learns from one load whether its row has any there.
constexpr int kStripColumns = 64, kStripBits = 10;
constexpr uint32_t kStripMost = 63;
struct Entry {
    int32_t id, place;                                   // id, and the entry's place in its row
};
struct Tempered {
    static constexpr bool kTargets = false;
    struct Picks {
        const uint16_t *strips = nullptr;                // [tokens][pitch], or null: nothing is picked
        const Entry *entries = nullptr;                  // [tokens][count]
        const int32_t *token = nullptr;                  // of a row
        float *picked = nullptr;                         // [tokens][count]
        int64_t pitch = 0;
        int32_t count = 0;
        uint32_t blocks = 0;                             // few tokens: the first so many blocks take the products of entries' rows
        const int64_t *ids = nullptr;                    // [tokens][count]
        int64_t ignore = 0;
    };
    float inverse;                                       // 1 / temperature
    __device__ __forceinline__ float of(float z) const { return z * inverse; }
};

// The hardware's exp2 gives 0 below 2^-126; d of 16-bit types is formed from probabilities lifted by this much, which keeps those
// down to 2^-150, and the units of its factor take the lift out again.
constexpr int kLift = 24;
template <typename T>
constexpr int lift_of = sizeof(T) == 2 ? kLift : 0;

// exp(z - from), and 2^lift of it.  The binary32 calls take the library function (1 ulp): their results are held to binary32
// accuracy; for 16-bit types the hardware's exp2 is far below their own rounding.
// (`from` comes multiplied by log2 e: its rounding moves all terms of a row alike, by less than the rounding of the row's lse.)
template <typename T>
__device__ __forceinline__ float exp_from(float z, float from)
{
    if constexpr (sizeof(T) == 4) return expf(z - from);
    else return __builtin_amdgcn_exp2f(__builtin_fmaf(z, kLog2e, -(from * kLog2e)));
}
template <typename T>
__device__ __forceinline__ float lifted(float z, float from)
{
    if constexpr (sizeof(T) == 4) return expf(z - from);
    else return __builtin_amdgcn_exp2f(__builtin_fmaf(z, kLog2e, __builtin_fmaf(-from, kLog2e, float(kLift))));
}

// ---------------------------------------------------------------- the tokens that count, and rows into place

// The tokens that count are listed, in order, with their targets and factors, and their hidden states copied into rows of whole steps.
// A token takes part if its target is not `ignore` and (gradient) its factor is not 0; the products then run over that list alone.
//
// One launch does both: every block looks at all targets (a few loads per thread for some thousand tokens, against a launch's 3 us) for the
// number of tokens that count, of those ahead of its own, and the largest finite factor; then it lists and copies its own.  Blocks past the
// first list_blocks pad rows of the weight meanwhile, where these have to be (see HeadLayout::padded).
// 4096 tokens of 768 bfloat16 elements, 15 % of which count: 7.5 us; 8192 that all count, and are not copied: 9.2 us; 125 of 519 binary32
// elements and a weight of 1003 rows to pad: 7.5 us.  All of it is latency: a launch, two dependent loads, two barriers.
constexpr int kListThreads = 1024, kListWaves = kListThreads / 64, kListEach = 8;

struct Lists {
    int32_t *place, *target;
    float *base, *factor;
    int32_t *token;          // of a row; or null
};
template <typename T>
struct Padding {
    const T *src;
    T *dst;
    int64_t rows, width, pitch;
};

// A row of `width` elements, or (src null) of zeros, into a row of `pitch`, by `threads` threads.
template <typename T>
__device__ __forceinline__ void copy_row(const T *src, int64_t width, T *dst, int64_t pitch, int thread, int threads)
{
    constexpr int kPer = 16 / int(sizeof(T)), kAhead = 8;       // (eight loads on their way at a time)
    typedef T Vec __attribute__((ext_vector_type(kPer)));
    typedef Vec Anywhere __attribute__((aligned(sizeof(T))));
    for (int64_t from = int64_t(thread) * kPer; from < pitch; from += int64_t(threads) * kPer * kAhead) {
        Vec v[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; i++) {
            const int64_t k = from + int64_t(i) * threads * kPer;
            v[i] = Vec(T(0.f));
            if (!src || k >= width) continue;
            if (k + kPer <= width) v[i] = *reinterpret_cast<const Anywhere *>(src + k);
            else
                for (int e = 0; e < kPer; e++) v[i][e] = k + e < width ? src[k + e] : T(0.f);
        }
#pragma unroll
        for (int i = 0; i < kAhead; i++) {
            const int64_t k = from + int64_t(i) * threads * kPer;
            if (k < pitch) *reinterpret_cast<Vec *>(dst + k) = v[i];
        }
    }
}

// Sums of a pair of counts and the maximum of a value over a block, in every thread.
struct Totals {
    int32_t before, all;
    float top;
};
__device__ __forceinline__ Totals block_totals(Totals t, Totals *waves)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        t.before += __shfl_xor(t.before, d, 64);
        t.all += __shfl_xor(t.all, d, 64);
        t.top = fmaxf(t.top, __shfl_xor(t.top, d, 64));
    }
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = t;
    __syncthreads();
    t = waves[0];
#pragma unroll
    for (int w = 1; w < kListWaves; w++) {
        t.before += waves[w].before;
        t.all += waves[w].all;
        t.top = fmaxf(t.top, waves[w].top);
    }
    return t;
}

// outer: a factor of all gradients.  in_place: where every token counts, the products read the hidden states themselves (see Hidden) and nothing is copied.
// depth: rows past the last one are zeros up to a whole step of the products' summed axis.
template <typename T>
__global__ __launch_bounds__(kListThreads) void list_tokens(const int64_t *__restrict__ targets, const float *__restrict__ dloss,
                                                            const float *__restrict__ lse, int64_t tokens, int64_t ignore, int64_t vocab,
                                                            int32_t top_bits, float outer, const T *__restrict__ hidden, int64_t width, T *__restrict__ rows,
                                                            int64_t pitch, int32_t depth, int32_t in_place, Header *header, Lists lists,
                                                            uint32_t list_blocks, Padding<T> weight)
{
    __shared__ Totals totals[kListWaves];
    __shared__ int32_t ahead[kListWaves], listed[kListThreads];
    const int tid = int(threadIdx.x), lane = tid & 63, wave = tid >> 6;
    if (blockIdx.x >= list_blocks) {
        for (int64_t row = int64_t(blockIdx.x - list_blocks) * kListWaves + wave; row < weight.rows; row += int64_t(gridDim.x - list_blocks) * kListWaves)
            copy_row(weight.src + row * weight.width, weight.width, weight.dst + row * weight.pitch, weight.pitch, lane, 64);
        return;
    }
    const int64_t each = (tokens + list_blocks - 1) / list_blocks, first = int64_t(blockIdx.x) * each;
    const int64_t end = first + each < tokens ? first + each : tokens;
    const auto counts = [&](int64_t t) { return targets[t] != ignore && (!dloss || dloss[t] != 0.f); };
    Totals mine{0, 0, 0.f};
    for (int64_t from = 0; from < tokens; from += kListThreads * kListEach) {
        int64_t v[kListEach];
        float g[kListEach];
#pragma unroll
        for (int k = 0; k < kListEach; k++) {
            const int64_t t = from + k * kListThreads + tid;
            v[k] = t < tokens ? targets[t] : ignore;
            g[k] = dloss && t < tokens ? dloss[t] : 1.f;
        }
#pragma unroll
        for (int k = 0; k < kListEach; k++) {
            if (v[k] == ignore || g[k] == 0.f) continue;
            mine.all++;
            mine.before += from + k * kListThreads + tid < first;
            const float size = fabsf(g[k]);
            if (size < __builtin_inff()) mine.top = fmaxf(mine.top, size);       // (neither infinities nor NaN)
        }
    }
    const Totals t = block_totals(mine, totals);
    // d is held in units of the largest factor, times 2^top_bits.  With factors that are all alike (a mean over tokens) a target that has
    // no probability yet then is exactly -2^top_bits, and near 1 the rounding is at its finest: in units of 1 all targets of a call
    // would be off by the same rounding of the factor, and with them the whole gradient, by up to 2^-8.  In binary16, with 14, elements of d down to
    // 2^-28 (4e-9) of the largest factor stay normal numbers, those under 2^-39 are lost, and nothing overflows, whatever the loss scale: a token
    // whose factor is far below the largest one keeps fewer of its small probabilities.
    // A factor that is not finite makes its own token's d so; the unit comes from the others, whose dhidden is none the worse for it.
    const float unit = !top_bits || t.top == 0.f ? 1.f : fmaxf(t.top, 0x1p-100f);
    if (blockIdx.x == 0 && tid == 0) *header = Header{t.all, ldexpf(unit, -top_bits) * outer};
    const bool copies = !(in_place && t.all == tokens);
    int32_t done = t.before;
    for (int64_t from = first; from < end; from += kListThreads) {
        const int64_t at = from + tid;
        const bool in = at < end && counts(at);
        const uint64_t vote = __ballot(in);
        if (lane == 0) ahead[wave] = __popcll(vote);
        __syncthreads();
        int32_t before = __popcll(vote & ((uint64_t(1) << lane) - 1)), here = 0;
        for (int w = 0; w < kListWaves; w++) {
            before += w < wave ? ahead[w] : 0;
            here += ahead[w];
        }
        if (at < end) {
            const int32_t row = done + before;
            lists.place[at] = in ? row : -1;
            if (in) {
                const int64_t v = targets[at];
                const bool outside = v < 0 || v >= vocab;
                listed[before] = int32_t(at - from);
                lists.target[row] = outside ? -1 : int32_t(v);
                if (lists.token) lists.token[row] = int32_t(at);
                if (dloss) {
                    lists.base[row] = lse[at];
                    lists.factor[row] = outside ? __builtin_nanf("") : top_bits ? ldexpf(dloss[at] / unit, top_bits - kLift) : dloss[at];
                }
            }
        }
        __syncthreads();
        if (copies)
            for (int32_t k = wave; k < here; k += kListWaves)
                copy_row(hidden + (from + listed[k]) * width, width, rows + int64_t(done + k) * pitch, pitch, lane, 64);
        done += here;
    }
    if (copies && blockIdx.x == list_blocks - 1)
        for (int64_t row = done + wave; row < (int64_t(done) + depth - 1) / depth * depth; row += kListWaves)
            copy_row(static_cast<const T *>(nullptr), width, rows + row * pitch, pitch, lane, 64);
}

// The weight in rows of whole steps; a block per row.
template <typename T>
__global__ __launch_bounds__(256) void pad_rows(const T *__restrict__ src, int64_t width, T *__restrict__ dst, int64_t pitch)
{
    copy_row(src + int64_t(blockIdx.x) * width, width, dst + int64_t(blockIdx.x) * pitch, pitch, int(threadIdx.x), 256);
}

// The hidden states that the products read: the caller's where every token counts and their rows fit the tiles as they are.
template <typename T>
struct Hidden {
    const T *own;            // or null: never
    const T *listed;
    int64_t tokens;
    __device__ __forceinline__ const T *of(int64_t count) const { return own && count == tokens ? own : listed; }
};

// The tokens of a loss call: listed, or as they come.  Few tokens or few logits take the same time whether all of them count or not, and
// need no list (a launch of 6 us beside 18 us for one token's logits); tokens that do not count get a loss of 0 in the end.
struct Tokens {
    const Header *header;    // null: as they come
    const int32_t *place, *target;
    const int64_t *targets;
    int64_t tokens, ignore, vocab;
    __device__ __forceinline__ int64_t count() const { return header ? header->count : tokens; }
    __device__ __forceinline__ int32_t row_of(int64_t token) const { return header ? place[token] : targets[token] == ignore ? -1 : int32_t(token); }
    __device__ __forceinline__ int32_t target_of(int64_t row) const
    {
        if (header) return target[row];
        const int64_t v = targets[row];
        return v < 0 || v >= vocab ? -1 : int32_t(v);
    }
};

// ---------------------------------------------------------------- logits

__host__ __device__ __forceinline__ uint32_t up(int64_t v, int to) { return uint32_t((v + to - 1) / to); }

template <typename K>
using Lds = unsigned char[K::kLds];

// Picks a tile's logits at its rows' entries.  Most rows have no entry among a wave's 64 columns, or one, anywhere, and registers have no index: so
// a wave that has any puts its logits into LDS, as many rows as its share of that holds, and each lane looks up one row's.  The loads that depend on each
// other are spread over the tile's end: where a row's entries are when it begins, the first two of them half way through the exponentials.
// Tiles with and without picking, us: 8192 x 2048 x 50257 bfloat16, 64 entries, 1292 and 1257; 4096 x 1024 x 50257 binary16, 128, 415 and 383; 615 x 768 x
// 30522, 32, 51 and 47.  Picking from the registers, by comparing each of a lane's sixteen columns: 1350, 449 and 56.
template <typename K, typename S>
struct Picker {
    __device__ __forceinline__ Picker(const typename S::Picks &, const K &, const Tokens &, int64_t, int64_t, int64_t) {}
    __device__ __forceinline__ void fetch(const typename S::Picks &) {}
    __device__ __forceinline__ void put(const typename S::Picks &, const K &, unsigned char *) {}
};
template <typename K>
struct Picker<K, Tempered> {
    using Picks = Tempered::Picks;
    static constexpr int kRowBytes = kStripColumns * 4, kShare = K::kLds / (K::WM * K::WN);
    static constexpr int kRows = 16 * K::TM < kShare / kRowBytes ? 16 * K::TM : kShare / kRowBytes, kRounds = 16 * K::TM / kRows;
    static_assert(K::TN * 16 == kStripColumns && kRows % 16 == 0 && kRows <= 64 && kRows * kRounds == 16 * K::TM, "a strip's rows in whole rounds");
    typedef int32_t Pair __attribute__((ext_vector_type(4)));              // two entries
    typedef Pair Anywhere __attribute__((aligned(8)));
    uint32_t at[kRounds];
    int32_t token[kRounds], column;
    Pair pair[kRounds];
    // first: the tile's first column in the vocabulary.
    __device__ __forceinline__ Picker(const Picks &picks, const K &tile, const Tokens &tokens, int64_t m0, int64_t count, int64_t first)
    {
        if (!picks.strips) return;
        const int64_t strip = (first + tile.wn) / kStripColumns;
        column = int32_t(strip * kStripColumns);
#pragma unroll
        for (int q = 0; q < kRounds; q++) {
            const int64_t row = m0 + tile.wm + q * kRows + tile.lane;
            const bool none = tile.lane >= kRows || row >= count || column >= tokens.vocab;      // (tiles go over both ends)
            token[q] = none ? 0 : count == tokens.tokens ? int32_t(row) : picks.token[row];
            at[q] = none ? 0 : picks.strips[token[q] * picks.pitch + strip];
        }
    }
    __device__ __forceinline__ static const Entry *row_of(const Picks &picks, int32_t token) { return picks.entries + int64_t(token) * picks.count; }
    // (the array is padded by two entries)
    __device__ __forceinline__ static Pair load(const Entry *p) { return *reinterpret_cast<const Anywhere *>(p); }
    __device__ __forceinline__ void fetch(const Picks &picks)
    {
        if (!picks.strips) return;
#pragma unroll
        for (int q = 0; q < kRounds; q++)
            if (at[q] >> kStripBits) pair[q] = load(row_of(picks, token[q]) + (at[q] & ((1u << kStripBits) - 1)));
    }
    static __device__ __forceinline__ void fence()
    {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");           // (LDS accesses of a wave are in order)
        __builtin_amdgcn_wave_barrier();
    }
    // lds: what the whole block is done with.  Its 16-byte pieces are permuted within a row, so that neighbouring rows' fall on different banks.
    __device__ __forceinline__ void put(const Picks &picks, const K &tile, unsigned char *lds)
    {
        if (!picks.strips) return;
        unsigned char *const own = lds + tile.wave * kShare;
        const int g = tile.lane >> 4, r = tile.lane & 15;
#pragma unroll
        for (int q = 0; q < kRounds; q++) {
            uint32_t left = at[q] >> kStripBits;
            if (!__ballot(left != 0)) continue;
#pragma unroll
            for (int i = 0; i < kRows / 16; i++)
#pragma unroll
                for (int j = 0; j < K::TN; j++)
                    *reinterpret_cast<f32x4 *>(own + (16 * i + r) * kRowBytes + (((4 * g + j) ^ r) << 4)) = tile.acc[q * (kRows / 16) + i][j];
            fence();
            uint32_t from = at[q] & ((1u << kStripBits) - 1);
            const bool more = left == kStripMost;
            if (more) left = uint32_t(picks.count) - from;       // (up to the end of the row, or of the strip)
            const Entry *const row = row_of(picks, token[q]);
            float *const out = picks.picked + int64_t(token[q]) * picks.count;
            const auto logit = [&](int32_t d) { return *reinterpret_cast<const float *>(own + tile.lane * kRowBytes + (((d >> 2) ^ r) << 4) + (d & 3) * 4); };
            Pair e = pair[q];
            while (left) {
                const Pair next = left > 2 ? load(row + from + 2) : e;
                const int32_t d = e[0] - column, d2 = e[2] - column;
                if (d >= 0 && d < kStripColumns) out[e[1]] = logit(d);
                if (left > 1 && d2 >= 0 && d2 < kStripColumns) out[e[3]] = logit(d2);
                if (left <= 2 || (more && d2 >= kStripColumns)) break;
                left -= 2;
                from += 2;
                e = next;
            }
            fence();
        }
    }
};

// Logits of a tile, and what its rows add to their softmax: the largest logit m, the sum of exp(logit - m), in binary32; parts join by
// m = max m_k, sum = sum_k sum_k exp(m_k - m), so that no logit is ever stored.  A lane holds 16 neighbouring columns of a row (strips),
// so a row's maximum and sum take two exchanges between lanes and one between waves.
// Bound by the matrix cores: 8192 x 2048 x 50257 bfloat16 1290 us = 1.31 PFLOP/s (the library's product of this shape 1.23), which
// issue in 0.63 of the cycles; without exponentials, maxima and stores it takes 0.95 of that time.  Sixteen steps per tile leave more of its
// ends uncovered: 4096 x 1024 x 50257 binary16 419 us = 1.01 PFLOP/s (the library's 0.86).  binary32, 509 x 768 x 30522: 205 us =
// 117 TFLOP/s of 154 in single passes, 180 us back to back.  With few tokens by reading W: 32 x 2048 x 50257 34 us from the memory-side cache,
// about 50 from memory.
template <typename K, typename S>
__global__ __launch_bounds__(K::kThreads, 2) void loss_tiles(Tokens tokens, Hidden<typename K::T> hidden, const typename K::T *weight,
                                                          int64_t pitch, int64_t first, int64_t columns, int64_t parts,
                                                          float2 *__restrict__ stats, float *__restrict__ picked, S softmax, typename S::Picks picks)
{
    using T = typename K::T;
    __shared__ __align__(256) Lds<K> lds;
    const int64_t count = tokens.count();
    int tm, tn;
    if (!tile_of_block(blockIdx.x, ~0u, up(count, K::BM), up(columns, K::BN), tm, tn)) return;
    const int64_t m0 = int64_t(tm) * K::BM, n0 = int64_t(tn) * K::BN;
    K tile;
    typename K::A a;
    typename K::B b;
    a.start(hidden.of(count), pitch, m0, count - m0, 0, int(threadIdx.x));
    b.start(weight, pitch, n0, columns - n0, 0, int(threadIdx.x));
    tile.run(a, b, int(pitch / K::kDepth), K::kDepth, lds);

    __syncthreads();
    float2 *joined = reinterpret_cast<float2 *>(lds);        // [WN][BM]
    const int g = tile.lane >> 4, r = tile.lane & 15, wave_n = tile.wave % K::WN;
    const int64_t c0 = n0 + tile.wn + 16 * g;
    const bool whole = n0 + K::BN <= columns;
    Picker<K, S> picker(picks, tile, tokens, m0, count, first + n0);
#pragma unroll
    for (int i = 0; i < K::TM; i++) {
        if (i == K::TM / 2) picker.fetch(picks);
        const int m = tile.wm + 16 * i + r;
        const int64_t row = m0 + m;
        if (S::kTargets && row < count) {
            const int64_t d = int64_t(tokens.target_of(row)) - first - c0;
            if (d >= 0 && d < 16) {
#pragma unroll
                for (int j = 0; j < K::TN; j++)
#pragma unroll
                    for (int e = 0; e < 4; e++)
                        if (d == 4 * j + e) picked[row] = tile.acc[i][j][e];
            }
        }
        float top = -__builtin_inff();
#pragma unroll
        for (int j = 0; j < K::TN; j++)
#pragma unroll
            for (int e = 0; e < 4; e++) {
                if (!whole && c0 + 4 * j + e >= columns) tile.acc[i][j][e] = -__builtin_inff();
                top = fmaxf(top, tile.acc[i][j][e]);
            }
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        top = softmax.of(top);                           // (a positive factor: the largest stays the largest)
        const float from = top == -__builtin_inff() ? 0.f : top;
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < K::TN; j++)
#pragma unroll
            for (int e = 0; e < 4; e++) sum += exp_from<T>(softmax.of(tile.acc[i][j][e]), from);
        sum += __shfl_xor(sum, 16, 64);
        sum += __shfl_xor(sum, 32, 64);
        if (g == 0) joined[wave_n * K::BM + m] = float2{top, sum};
    }
    __syncthreads();
    for (int m = int(threadIdx.x); m < K::BM; m += K::kThreads) {
        if (m0 + m >= count) break;
        float top = joined[m].x;
#pragma unroll
        for (int w = 1; w < K::WN; w++) top = fmaxf(top, joined[w * K::BM + m].x);
        const float from = top == -__builtin_inff() ? 0.f : top;
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < K::WN; w++) sum += joined[w * K::BM + m].y * __builtin_amdgcn_exp2f((joined[w * K::BM + m].x - from) * kLog2e);
        stats[(m0 + m) * parts + (first + n0) / K::BN] = float2{top, sum};
    }
    if constexpr (!S::kTargets) __syncthreads();
    picker.put(picks, tile, lds);
}

// The student's logits at some entries of a token, by a wave: the products of its hidden state and the weight's rows, kDots rows on their way at a
// time.  `out(k, id, inside, z)` is called by all lanes.
template <typename T>
struct Slice {               // 16 bytes of a row that starts at any element, as binary32
    static constexpr int V = 16 / int(sizeof(T));
    float v[V];
    __device__ __forceinline__ void load(const T *row, int64_t column, int64_t width)
    {
        typedef T Vec __attribute__((ext_vector_type(V)));
        typedef Vec Anywhere __attribute__((aligned(sizeof(T))));
        if (column + V <= width) {
            const Vec x = *reinterpret_cast<const Anywhere *>(row + column);
#pragma unroll
            for (int e = 0; e < V; e++) v[e] = float(x[e]);
        } else {
#pragma unroll
            for (int e = 0; e < V; e++) v[e] = column + e < width ? float(row[column + e]) : 0.f;
        }
    }
};
constexpr int kDots = 4;
template <typename T, class Out>
__device__ __forceinline__ void entry_dots(const T *x, const T *weight, int64_t width, int64_t vocab, const int64_t *ids, int64_t ignore, int from, int count,
                                           int lane, Out out)
{
    int64_t id[kDots];
    bool inside[kDots];
    float dot[kDots];
#pragma unroll
    for (int k = 0; k < kDots; k++) {
        id[k] = from + k < count ? ids[from + k] : ignore;
        inside[k] = id[k] != ignore && id[k] >= 0 && id[k] < vocab;
        dot[k] = 0.f;
    }
    for (int64_t column = lane * Slice<T>::V; column < width; column += 64 * Slice<T>::V) {
        Slice<T> a, b[kDots];
        a.load(x, column, width);
#pragma unroll
        for (int k = 0; k < kDots; k++) b[k].load(weight + (inside[k] ? id[k] : 0) * width, column, width);
#pragma unroll
        for (int k = 0; k < kDots; k++)
#pragma unroll
            for (int e = 0; e < Slice<T>::V; e++) dot[k] = __builtin_fmaf(a.v[e], b[k].v[e], dot[k]);
    }
#pragma unroll
    for (int k = 0; k < kDots; k++) {
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) dot[k] += __shfl_xor(dot[k], d, 64);
        if (from + k < count) out(from + k, id[k], inside[k], dot[k]);
    }
}

// The same for few tokens, where reading W is all that takes time, and for few logits: a block per 16 tokens and kFewColumns rows of W, whose four waves each sum a
// quarter of the width.  W goes from memory to the registers of the one wave that uses it, a unit of 128 bytes per row ahead of the products,
// so there are no barriers on the way and every wave has its own loads in flight; tokens are read from the caches, at half of W's bytes.
// Calls with it and with tiny tiles, us: 1 x 2048 x 50257 bfloat16 (206 MB) 44 and 56, 1 x 4096 x 50257 82 and 96, 16 x 2048 x 50257 48 and 60,
// 16 x 768 x 30522 binary32 28 and 38; 103 MB that the memory-side cache partly holds 23 and 22, that it does not 25 and 27.  For 32 and 64
// tokens the same with two and four times the tokens per wave was slower than the tiles (206 MB 62 and 62, 84 and 62): tokens then cost as
// many bytes of the caches as W or more.  32 columns a block: 16 and 64 took 59 and 51 instead of 49 for 16 x 2048 x 50257.
constexpr int kFewWaves = 4, kFewPitch = kFewColumns + 4;
// What a wave's quarter of the width adds to the logits of `count` rows of hidden states (at most 16 are looked at) and `columns` of the weight.
template <typename T>
__device__ __forceinline__ void few_products(float (&part)[kFewWaves][16][kFewPitch], const T *__restrict__ hidden, const T *__restrict__ weight, int64_t width,
                                             int columns, int count, int wave, int lane)
{
    using E = Element<T>;
    using Frag = typename E::Frag;
    typedef Frag Anywhere __attribute__((aligned(sizeof(T))));         // (rows start at any element)
    constexpr int TN = kFewColumns / 16, kUnit = kStepBytes / int(sizeof(T));
    const int g = lane >> 4, r = lane & 15;
    // (rows past the last one are read from it, and not used)
    uint32_t of_column[TN];
    const uint32_t of_token = uint32_t(r < count ? r : count - 1) * uint32_t(width * sizeof(T)) + g * 16;
#pragma unroll
    for (int j = 0; j < TN; j++) of_column[j] = uint32_t(16 * j + r < columns ? 16 * j + r : columns - 1) * uint32_t(width * sizeof(T)) + g * 16;
    struct Unit {
        Frag a[2], b[2][TN];
    };
    const int units = int(width / kUnit), from = units * wave / kFewWaves, to = units * (wave + 1) / kFewWaves;
    const unsigned char *w = reinterpret_cast<const unsigned char *>(weight), *x = reinterpret_cast<const unsigned char *>(hidden);
    const auto load = [&](Unit &u, int at) {
#pragma unroll
        for (int half = 0; half < 2; half++)
#pragma unroll
            for (int j = 0; j < TN; j++) u.b[half][j] = *reinterpret_cast<const Anywhere *>(w + int64_t(at) * kStepBytes + half * (kStepBytes / 2) + of_column[j]);
#pragma unroll
        for (int half = 0; half < 2; half++)
            u.a[half] = *reinterpret_cast<const Anywhere *>(x + int64_t(at) * kStepBytes + half * (kStepBytes / 2) + of_token);
    };
    f32x4 acc[TN];
#pragma unroll
    for (int j = 0; j < TN; j++) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const auto multiply = [&](const Unit &u) {
#pragma unroll
        for (int half = 0; half < 2; half++)
#pragma unroll
            for (int j = 0; j < TN; j++) acc[j] = E::mfma(u.b[half][j], u.a[half], acc[j]);
    };
    if (from < to) {
        Unit u0, u1;
        load(u0, from);
        int at = from;
        for (; at + 2 < to; at += 2) {
            load(u1, at + 1);
            __builtin_amdgcn_sched_barrier(0);
            multiply(u0);
            __builtin_amdgcn_sched_barrier(0);
            load(u0, at + 2);
            __builtin_amdgcn_sched_barrier(0);
            multiply(u1);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (at + 1 < to) load(u1, at + 1);
        multiply(u0);
        if (at + 1 < to) multiply(u1);
    }
    const int rest = int(width % kUnit);
    if (rest && wave == kFewWaves - 1) {                 // the width's last, partial unit
        Unit u;
        const auto load_rest = [&](const unsigned char *p, int half) {
            Frag v;
#pragma unroll
            for (int e = 0; e < 16 / int(sizeof(T)); e++)
                v[e] = half * (kUnit / 2) + g * (16 / int(sizeof(T))) + e < rest ? reinterpret_cast<const T *>(p)[e] : T(0.f);
            return v;
        };
#pragma unroll
        for (int half = 0; half < 2; half++) {
            const int64_t at = int64_t(units) * kStepBytes + half * (kStepBytes / 2);
#pragma unroll
            for (int j = 0; j < TN; j++) u.b[half][j] = load_rest(w + at + of_column[j], half);
            u.a[half] = load_rest(x + at + of_token, half);
        }
        multiply(u);
    }
#pragma unroll
    for (int j = 0; j < TN; j++) *reinterpret_cast<f32x4 *>(&part[wave][r][16 * j + 4 * g]) = acc[j];
}

template <typename T, typename S>
__global__ __launch_bounds__(64 * kFewWaves, 4) void few_tiles(Tokens tokens, const T *__restrict__ hidden, const T *__restrict__ weight,
                                                               int64_t width, uint32_t groups, int64_t parts, float2 *__restrict__ stats,
                                                               float *__restrict__ picked, S softmax, typename S::Picks picks)
{
    __shared__ __align__(16) float part[kFewWaves][16][kFewPitch];
    const int tid = int(threadIdx.x), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    uint32_t at_block = blockIdx.x;
    if constexpr (!S::kTargets) {
        if (at_block < picks.blocks) {                   // (their products take a few dependent loads, so they go ahead of W)
            const int64_t item = int64_t(at_block) * kFewWaves + wave, each = (picks.count + kDots - 1) / kDots, token = item / each;
            if (token >= tokens.tokens) return;
            float *const out = picks.picked + token * picks.count;
            entry_dots(hidden + token * width, weight, width, tokens.vocab, picks.ids + token * picks.count, picks.ignore, int(item % each) * kDots,
                       picks.count, lane, [&](int k, int64_t, bool, float z) { if (lane == 0) out[k] = z; });
            return;
        }
        at_block -= picks.blocks;
    }
    const uint32_t block = at_block / groups;
    const int64_t n0 = int64_t(block) * kFewColumns, m0 = int64_t(at_block % groups) * kFewTokens;
    const int columns = int(tokens.vocab - n0 < kFewColumns ? tokens.vocab - n0 : kFewColumns), count = int(tokens.tokens - m0);
    few_products(part, hidden + m0 * width, weight + n0 * width, width, columns, count, wave, lane);
    __syncthreads();
    // a token's columns: kLanes neighbouring lanes, kEach columns a lane
    constexpr int kEach = 16 * kFewColumns / (64 * kFewWaves), kLanes = kFewColumns / kEach;
    const int m = tid / kLanes, first = tid % kLanes * kEach;
    const int32_t target = S::kTargets && m < count ? tokens.target_of(m0 + m) : -1;
    float z[kEach], top = -__builtin_inff();
#pragma unroll
    for (int e = 0; e < kEach; e++) {
        z[e] = 0.f;
#pragma unroll
        for (int k = 0; k < kFewWaves; k++) z[e] += part[k][m][first + e];
        if (S::kTargets && m < count && target == n0 + first + e) picked[m0 + m] = z[e];
        z[e] = softmax.of(z[e]);
        if (first + e >= columns) z[e] = -__builtin_inff();
        top = fmaxf(top, z[e]);
    }
#pragma unroll
    for (int d = kLanes / 2; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
    const float base = top == -__builtin_inff() ? 0.f : top;
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < kEach; e++) sum += exp_from<T>(z[e], base);
#pragma unroll
    for (int d = kLanes / 2; d > 0; d >>= 1) sum += __shfl_xor(sum, d, 64);
    if (m < count && first == 0) stats[(m0 + m) * parts + block] = float2{top, sum};
}

// The logarithm of a row's sum of exponentials from its parts, by WAVES waves; in every lane of theirs.
template <int WAVES>
__device__ __forceinline__ float log_sum(const float2 *__restrict__ s, int64_t parts, int lane)
{
    constexpr int kLanes = 64 * WAVES;
    float top = -__builtin_inff(), sum = 0.f;
    for (int64_t first = 0; first < parts; first += 4 * kLanes) {
        float2 v[4];
#pragma unroll
        for (int k = 0; k < 4; k++) {
            const int64_t p = first + kLanes * k + lane;
            v[k] = p < parts ? s[p] : float2{-__builtin_inff(), 0.f};
        }
        float most = top;
#pragma unroll
        for (int k = 0; k < 4; k++) most = fmaxf(most, v[k].x);
        const float from = most == -__builtin_inff() ? 0.f : most;
        sum *= expf(top - from);
#pragma unroll
        for (int k = 0; k < 4; k++) sum += v[k].y * expf(v[k].x - from);
        top = most;
    }
    const auto join = [&](int width) {
        float all = top;
        for (int d = width / 2; d > 0; d >>= 1) all = fmaxf(all, __shfl_xor(all, d, 64));
        const float from = all == -__builtin_inff() ? 0.f : all;
        sum *= expf(top - from);
        for (int d = width / 2; d > 0; d >>= 1) sum += __shfl_xor(sum, d, 64);
        top = all;
    };
    join(64);
    if constexpr (WAVES > 1) {
        __shared__ float2 waves[WAVES];
        if ((lane & 63) == 0) waves[lane >> 6] = float2{top, sum};
        __syncthreads();
        const float2 v = waves[lane % WAVES];
        top = v.x;
        sum = v.y;
        join(WAVES);
    }
    return (top == -__builtin_inff() ? 0.f : top) + logf(sum);
}

// Joins the parts of every token's softmax: a wave per token, four of them in a block, or (few tokens) a block of many waves per token.
// 8192 tokens of 197 parts: 6.4 us (12.9 MB, 2 TB/s); one token of 1571 parts: 3.9 us, a launch and two rounds of loads.
constexpr int kJoinWaves = 16;
template <int WAVES>
constexpr int join_tokens = WAVES > 1 ? 1 : 4;
template <int WAVES>
__global__ __launch_bounds__(64 * WAVES * join_tokens<WAVES>) void join_loss(Tokens tokens, int64_t parts, int64_t pitch, const float2 *__restrict__ stats,
                                                             const float *__restrict__ picked, float *__restrict__ loss, float *__restrict__ lse)
{
    constexpr int kLanes = 64 * WAVES;
    const int lane = int(threadIdx.x) % kLanes;
    const int64_t token = int64_t(blockIdx.x) * join_tokens<WAVES> + threadIdx.x / kLanes;
    const int32_t row = token < tokens.tokens ? tokens.row_of(token) : -1;
    if (row < 0) {                                       // (for WAVES > 1, the whole block's row)
        if (token < tokens.tokens && lane == 0) loss[token] = lse[token] = 0.f;
        return;
    }
    const float total = log_sum<WAVES>(stats + row * pitch, parts, lane);
    if (lane != 0) return;
    lse[token] = total;
    loss[token] = tokens.target_of(row) < 0 ? __builtin_nanf("") : total - picked[row];
}

// ---------------------------------------------------------------- gradient

// From the upper parts of d to the lower ones, in rows: whole tiles of 64, and whole steps of the products that sum over them.
__host__ __device__ __forceinline__ int64_t lower_rows(int64_t count) { return (count + 63) / 64 * 64; }

// d in two parts of fewer bits.  The compiler may round a product to binary16 in one step for one use of it, and by way of binary32 for another:
// where that makes a difference (one element in some ten thousand) the parts would be those of two numbers, a step of the upper one apart.
// So d is a number in a register first.
template <typename D>
struct TwoParts {
    D upper, rest;
    explicit __device__ __forceinline__ TwoParts(float d)
    {
        asm("" : "+v"(d));
        upper = D(d);
        rest = D(d - float(upper));
    }
};

// What the last blocks of d's launch do besides tiles: nothing, or another kernel's work that the products after d need.  It fills the compute units that the
// last round of tiles leaves idle.
struct Nothing {
    static constexpr bool kAny = false;
    uint32_t blocks = 0;
};

// d of a tile of a piece: logits as above, then dloss (exp(z - lse) - [v = target]) in its units, in the operands' type.
// Every element of the piece's whole tiles is written; those of no token or no column are zeros.
// d is rounded to the operands' type once, because the products that follow read it from the matrix cores' operands: its relative error,
// half a unit of that type, is what the results are rounded to as well.  Gradients of partly trained heads (8192 and 4096 tokens before 30522 and
// 50257 columns) are 1.07 to 1.11 times as far from the exact ones as these rounded to bfloat16, 1.17 times in binary16, all of it from the
// one element of a row that is its target's; d in two parts would take that away for 4 N V H more operations.
// Forming the logits again costs 2 N V H operations and saves 4 N V bytes written and read by the loss and N V bytes of workspace that would have
// to live from one call to the other.
// 8192 tokens x 2048 x 25344 columns, bfloat16: 709 us = 1.20 PFLOP/s, with 0.41 GB written at the tiles' ends while no products run.
//
// D: the type that d is held in, where that is not the operands' (see Calls).  LOWER: what rounding takes from d is held as well, lower_rows(count) rows on.
// BESIDE: what the launch's last blocks do instead of tiles (see Nothing).
template <typename K, typename S, typename D, bool LOWER, typename BESIDE>
__global__ __launch_bounds__(K::kThreads, 2) void delta_tiles(const Header *header, Hidden<typename K::T> hidden, const typename K::T *weight,
                                                           int64_t pitch, int64_t first, int64_t columns,
                                                           const int32_t *__restrict__ target, const float *__restrict__ lse,
                                                           const float *__restrict__ factor, D *__restrict__ delta, int64_t piece, S softmax,
                                                           BESIDE beside)
{
    using T = typename K::T;
    if constexpr (BESIDE::kAny) {
        const uint32_t of_tiles = gridDim.x - beside.blocks;
        if (blockIdx.x >= of_tiles) {
            beside(blockIdx.x - of_tiles, header, hidden, weight, pitch);
            return;
        }
    }
    __shared__ __align__(256) Lds<K> lds;
    const int64_t count = header->count, lower = lower_rows(count);
    int tm, tn;
    if (!tile_of_block(blockIdx.x, ~0u, up(count, K::BM), up(columns, K::BN), tm, tn)) return;
    const int64_t m0 = int64_t(tm) * K::BM, n0 = int64_t(tn) * K::BN;
    K tile;
    typename K::A a;
    typename K::B b;
    a.start(hidden.of(count), pitch, m0, count - m0, 0, int(threadIdx.x));
    b.start(weight, pitch, n0, columns - n0, 0, int(threadIdx.x));
    tile.run(a, b, int(pitch / K::kDepth), K::kDepth, lds);

    // Few instructions per element: this runs while the matrix cores idle.  The one element of a row that is the target's is written
    // again afterwards, by the same lane.
    const int g = tile.lane >> 4, r = tile.lane & 15;
    const int64_t c0 = n0 + tile.wn + 16 * g;
    const bool whole = m0 + K::BM <= count && n0 + K::BN <= columns;
    constexpr int kPer = 16 / int(sizeof(D));
    typedef D Vec __attribute__((ext_vector_type(kPer)));
#pragma unroll
    for (int i = 0; i < K::TM; i++) {
        const int64_t row = m0 + tile.wm + 16 * i + r;
        const float base = row < count ? lse[row] : 0.f, f = row < count ? factor[row] : 0.f;
        const bool counts = row < count && (S::kTargets || f != 0.f);          // (few tokens are not listed: some may take no part)
        const int64_t hit = S::kTargets && counts ? int64_t(target[row]) - first - c0 : -1;
        D *const out = delta + row * piece + c0;
#pragma unroll
        for (int k = 0; k < 16; k += kPer) {
            Vec v, rest;
#pragma unroll
            for (int e = 0; e < kPer; e++) {
                const float d = lifted<T>(softmax.of(tile.acc[i][(k + e) / 4][(k + e) % 4]), base) * f;
                if constexpr (LOWER) {
                    const TwoParts<D> parts(d);
                    v[e] = parts.upper;
                    rest[e] = parts.rest;
                } else v[e] = D(d);
            }
            if (!whole || (!S::kTargets && !counts))
#pragma unroll
                for (int e = 0; e < kPer; e++)
                    if (!counts || c0 + k + e >= columns) {
                        v[e] = D(0.f);
                        if (LOWER) rest[e] = D(0.f);
                    }
            *reinterpret_cast<Vec *>(out + k) = v;
            if (LOWER) *reinterpret_cast<Vec *>(out + lower * piece + k) = rest;
        }
        if (S::kTargets && hit >= 0 && hit < 16) {
            float z = 0.f;
#pragma unroll
            for (int k = 0; k < 16; k++)
                if (hit == k) z = tile.acc[i][k / 4][k % 4];
            out[hit] = D((lifted<T>(z, base) - float(1 << lift_of<T>)) * f);
        }
    }
}

// Into how many parts the sum over a piece is split, so that the tiles of few tokens fill the chip too: as many as `blocks` allow,
// of at least kLeastSteps steps.  Each part has sums of its own, joined by round_hidden in order.
constexpr int kLeastSteps = 8;
__host__ __device__ __forceinline__ uint32_t parts_of(uint32_t tiles, uint32_t steps, uint32_t blocks)
{
    const uint32_t most = steps / kLeastSteps, parts = tiles ? blocks / tiles : 1;
    return parts < 1 || most < 1 ? 1 : parts < most ? parts : most;
}

// The sum of the parts, in order, with eight of them on their way at a time.
__device__ __forceinline__ f32x4 joined(const float *first, int64_t apart, uint32_t parts)
{
    f32x4 v{0.f, 0.f, 0.f, 0.f};
    for (uint32_t p = 0; p < parts; p += 8) {
        f32x4 x[8];
#pragma unroll
        for (uint32_t k = 0; k < 8; k++)
            x[k] = p + k < parts ? *reinterpret_cast<const f32x4 *>(first + int64_t(p + k) * apart) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (uint32_t k = 0; k < 8; k++) v += x[k];
    }
    return v;
}

// dx += d W over a piece, in binary32.  accumulate: not the first piece.  W is read along its rows, as stored; the matrix cores want its
// columns, and transposing LDS reads give them (Side::fragment).  8192 x 25344 columns x 2048, bfloat16: 616 us = 1.38 PFLOP/s.
// SCALED: the product is also multiplied by *scale.
template <typename K, bool SCALED>
__device__ __forceinline__ void hidden_block(unsigned char *lds, uint32_t block, const Header *header, const typename K::T *delta, int64_t piece,
                                             const typename K::T *weight, int64_t pitch, int64_t columns, int32_t blocks, int32_t accumulate,
                                             float *__restrict__ sums, const float *scale)
{
    const int64_t count = header->count;
    const uint32_t tiles_m = up(count, K::BM), tiles_n = up(pitch, K::BN), parts = parts_of(tiles_m * tiles_n, up(piece, K::kDepth), blocks);
    int tm, tn;
    // the parts of a tile are as far apart as possible, the tiles of a part neighbours
    if (!tile_of_block(block, ~0u, tiles_m * parts, tiles_n, tm, tn)) return;
    const uint32_t part = uint32_t(tm) / tiles_m;
    const int64_t m0 = int64_t(tm - part * tiles_m) * K::BM, n0 = int64_t(tn) * K::BN;
    const uint32_t all = up(columns, K::kDepth), each = up(all, int(parts)), from = part * each;
    const int steps = int(from >= all ? 0 : all - from < each ? all - from : each);
    K tile;
    typename K::A a;
    typename K::B b;
    const int64_t k0 = steps ? int64_t(from) * K::kDepth : 0;
    a.start(delta, piece, m0, count - m0, k0, int(threadIdx.x));
    b.start(weight, pitch, n0, pitch - n0, k0, int(threadIdx.x));
    const int64_t left = columns - k0 - int64_t(steps - 1) * K::kDepth;
    tile.run(a, b, steps, int(left < K::kDepth ? left : K::kDepth), lds);
    const int g = tile.lane >> 4, r = tile.lane & 15;
    float *const own = sums + int64_t(part) * count * pitch;
    const float by = SCALED ? *scale : 1.f;
#pragma unroll
    for (int i = 0; i < K::TM; i++) {
        const int64_t row = m0 + tile.wm + 16 * i + r;
        if (row >= count) continue;
#pragma unroll
        for (int j = 0; j < K::TN; j++) {
            const int64_t column = n0 + tile.wn + 16 * j + 4 * g;
            if (column >= pitch) continue;
            f32x4 *p = reinterpret_cast<f32x4 *>(own + row * pitch + column);
            const f32x4 v = SCALED ? tile.acc[i][j] * by : tile.acc[i][j];
            *p = accumulate ? *p + v : v;
        }
    }
}

template <typename K, bool SCALED>
__global__ __launch_bounds__(K::kThreads, 2) void hidden_tiles(const Header *header, const typename K::T *delta, int64_t piece,
                                                            const typename K::T *weight, int64_t pitch, int64_t columns, int32_t blocks,
                                                            int32_t accumulate, float *__restrict__ sums, const float *scale)
{
    __shared__ __align__(256) Lds<K> lds;
    hidden_block<K, SCALED>(lds, blockIdx.x, header, delta, piece, weight, pitch, columns, blocks, accumulate, sums, scale);
}

// dW = d^T x for the rows of a piece.  The tiles fill the chip's compute units some number of times; those of the last, partial round are
// split over the tokens into as many parts as fill it, each part with sums of its own (`spare`, by part and tile), which weight_rest
// joins.  (Without that, 50257 x 2048 weights in two pieces took 4 rounds each for 3.06 rounds' work.)  Both operands are read along their
// rows and transposed on their way out of LDS.  25344 rows, 8192 tokens, width 2048, bfloat16: 653 us = 1.30 PFLOP/s, and 11 us of joining.
struct Rounds {
    uint32_t whole;          // tiles that a block computes alone
    uint32_t rest;           // tiles of the last round
    uint32_t parts;          // of each of these
};
__host__ __device__ __forceinline__ Rounds rounds_of(uint32_t tiles, uint32_t steps, uint32_t blocks)
{
    const uint32_t whole = tiles / blocks * blocks, rest = tiles - whole, most = steps / kLeastSteps;
    uint32_t parts = rest ? blocks / rest : 1;
    parts = parts < most ? parts : most;
    return parts < 2 ? Rounds{tiles, 0, 1} : Rounds{whole, rest, parts};
}

template <typename T>
__device__ __forceinline__ void store_weights(T *dweight, int64_t row, int64_t column, int64_t width, f32x4 v, float unscale)
{
    typedef T Four __attribute__((ext_vector_type(4)));
    Four out;
#pragma unroll
    for (int e = 0; e < 4; e++) out[e] = T(v[e] * unscale);
    typedef Four Anywhere __attribute__((aligned(sizeof(T))));          // (rows start at any element)
    T *p = dweight + row * width + column;
    if (column + 4 <= width) {
        *reinterpret_cast<Anywhere *>(p) = out;
    } else {
#pragma unroll
        for (int e = 0; e < 4; e++)
            if (column + e < width) p[e] = out[e];
    }
}

template <typename K, typename OUT, bool SCALED>
__device__ __forceinline__ void weight_block(unsigned char *lds, uint32_t block, const Header *header, const typename K::T *delta, int64_t piece,
                                             Hidden<typename K::T> hidden, int64_t pitch, int64_t columns, int64_t width, int32_t blocks,
                                             OUT *__restrict__ dweight, float *__restrict__ spare, const float *scale)
{
    const int64_t count = header->count;
    const uint32_t tiles_m = up(columns, K::BM), tiles_n = up(width, K::BN), all = up(count, K::kDepth);
    const Rounds r = rounds_of(tiles_m * tiles_n, all, uint32_t(blocks));
    uint32_t from = 0, steps = all, part = 0, tile_at = block;
    const bool shared = block >= r.whole;
    if (shared) {
        const uint32_t at = block - r.whole;
        if (at >= r.rest * r.parts) return;
        part = at / r.rest;
        tile_at = r.whole + at % r.rest;
        const uint32_t each = up(all, int(r.parts));
        from = part * each;
        steps = from >= all ? 0 : all - from < each ? all - from : each;
        if (!steps) from = 0;
    }
    int tm, tn;
    if (!tile_of_block(tile_at, r.whole, tiles_m, tiles_n, tm, tn)) return;
    const int64_t m0 = int64_t(tm) * K::BM, n0 = int64_t(tn) * K::BN;
    K tile;
    typename K::A a;
    typename K::B b;
    a.start(delta, piece, m0, piece - m0, int64_t(from) * K::kDepth, int(threadIdx.x));
    b.start(hidden.of(count), pitch, n0, pitch - n0, int64_t(from) * K::kDepth, int(threadIdx.x));
    tile.run(a, b, int(steps), K::kDepth, lds);
    const int g = tile.lane >> 4, l = tile.lane & 15;
    if (shared) {
        float *own = spare + int64_t(block - r.whole) * (K::BM * K::BN);
#pragma unroll
        for (int i = 0; i < K::TM; i++)
#pragma unroll
            for (int j = 0; j < K::TN; j++)
                *reinterpret_cast<f32x4 *>(own + (tile.wm + 16 * i + l) * K::BN + tile.wn + 16 * j + 4 * g) = tile.acc[i][j];
        return;
    }
    const float unscale = SCALED ? header->unscale * *scale : header->unscale;
#pragma unroll
    for (int i = 0; i < K::TM; i++) {
        const int64_t row = m0 + tile.wm + 16 * i + l;
        if (row >= columns) continue;
#pragma unroll
        for (int j = 0; j < K::TN; j++) {
            const int64_t column = n0 + tile.wn + 16 * j + 4 * g;
            if (column < width) store_weights(dweight, row, column, width, tile.acc[i][j], unscale);
        }
    }
}

template <typename K, typename OUT, bool SCALED>
__global__ __launch_bounds__(K::kThreads, 2) void weight_tiles(const Header *header, const typename K::T *delta, int64_t piece,
                                                            Hidden<typename K::T> hidden, int64_t pitch, int64_t columns, int64_t width,
                                                            int32_t blocks, OUT *__restrict__ dweight, float *__restrict__ spare,
                                                            const float *scale)
{
    __shared__ __align__(256) Lds<K> lds;
    weight_block<K, OUT, SCALED>(lds, blockIdx.x, header, delta, piece, hidden, pitch, columns, width, blocks, dweight, spare, scale);
}

// Both products of d in one launch, where both take small tiles and neither fills the chip: a launch's time less (125 x 519 x 1003 binary32
// 8.9 us instead of 8.4 and 5.9 one after the other, and what lies between launches).  us of whole gradients in two launches and in one: 128 x
// 512 x 1000 (128 tiles of the weight) binary32 28.6 and 23.5, bfloat16 27.4 and 22.6, binary16 27.3 and 22.7; 128 x 2048 x 2000 (1024, as many
// as blocks fit the chip: the limit) 62.4 and 60.9, 44.6 and 42.3, 44.7 and 42.4; x 4000 (2016) 94.7 and 90.2, 60.6 and 55.3, 62.5 and 55.9;
// x 8000 (4000) 128 and 124, alike in 16 bits, whose large tiles catch up there.
template <typename KH, typename KW>
__global__ __launch_bounds__(KH::kThreads, 2) void both_tiles(uint32_t of_hidden, const Header *header, const typename KH::T *delta, int64_t piece,
                                                           const typename KH::T *weight, int64_t pitch, int64_t columns, int32_t blocks,
                                                           int32_t accumulate, float *__restrict__ sums, Hidden<typename KH::T> hidden,
                                                           int64_t width, typename KH::T *__restrict__ dweight, float *__restrict__ spare)
{
    static_assert(KH::kThreads == KW::kThreads, "one launch");
    __shared__ __align__(256) unsigned char lds[KH::kLds > KW::kLds ? KH::kLds : KW::kLds];
    if (blockIdx.x < of_hidden) hidden_block<KH, false>(lds, blockIdx.x, header, delta, piece, weight, pitch, columns, blocks, accumulate, sums, nullptr);
    else weight_block<KW, typename KW::T, false>(lds, blockIdx.x - of_hidden, header, delta, piece, hidden, pitch, columns, width, blocks, dweight, spare, nullptr);
}

// The tiles of weight_tiles' last round from their parts: a block per 16 rows of a tile.
template <typename K, typename OUT, bool SCALED>
__global__ __launch_bounds__(256) void weight_rest(const Header *header, int64_t columns, int64_t width, int32_t blocks,
                                                   OUT *__restrict__ dweight, const float *__restrict__ spare, const float *scale)
{
    constexpr int kStrip = 16;
    const uint32_t tiles_m = up(columns, K::BM), tiles_n = up(width, K::BN);
    const Rounds r = rounds_of(tiles_m * tiles_n, up(header->count, K::kDepth), uint32_t(blocks));
    const uint32_t at = blockIdx.x / (K::BM / kStrip), strip = blockIdx.x % (K::BM / kStrip);
    int tm, tn;
    if (at >= r.rest || !tile_of_block(r.whole + at, r.whole, tiles_m, tiles_n, tm, tn)) return;
    const float unscale = SCALED ? header->unscale * *scale : header->unscale;
    for (int k = int(threadIdx.x) * 4; k < kStrip * K::BN; k += 1024) {
        const int m = int(strip) * kStrip + k / K::BN, n = k % K::BN;
        const int64_t row = int64_t(tm) * K::BM + m, column = int64_t(tn) * K::BN + n;
        if (row >= columns || column >= width) continue;
        const f32x4 v = joined(spare + int64_t(at) * (K::BM * K::BN) + m * K::BN + n, int64_t(r.rest) * (K::BM * K::BN), r.parts);
        store_weights(dweight, row, column, width, v, unscale);
    }
}

// dhidden from the sums, in their units; a block per token.  side, steps: of the kernel that left them.  Bound by memory: 8192 x 2048
// binary32 sums to bfloat16 23 us (101 MB, 4.4 TB/s); 4096 tokens of 768, the 15 % that
// count in 28 parts (their nine tiles, over 256 compute units: 53 MB), 12.5 us.
// LOWER: the header counts both parts' rows, and the sums of the lower part are half as many rows on.
template <typename T, bool LOWER>
__global__ __launch_bounds__(256) void round_hidden(const Header *header, const int32_t *__restrict__ place, const float *__restrict__ sums,
                                                    int64_t pitch, int64_t width, int32_t side, int32_t steps, int32_t blocks,
                                                    T *__restrict__ dhidden)
{
    typedef T Four __attribute__((ext_vector_type(4)));
    typedef Four Anywhere __attribute__((aligned(sizeof(T))));          // (rows start at any element)
    const int64_t token = blockIdx.x, count = header->count;
    const int32_t row = place[token];
    const float unscale = header->unscale;
    const uint32_t parts = parts_of(up(count, side) * up(pitch, side), uint32_t(steps), uint32_t(blocks));
    const float *s = sums + int64_t(row < 0 ? 0 : row) * pitch;
    T *d = dhidden + token * width;
    for (int64_t k = int64_t(threadIdx.x) * 4; k < width; k += 1024) {
        f32x4 v = row < 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : joined(s + k, count * pitch, parts);
        if (LOWER && row >= 0) v += joined(s + count / 2 * pitch + k, count * pitch, parts);
        Four out;
#pragma unroll
        for (int e = 0; e < 4; e++) out[e] = T(v[e] * unscale);
        if (k + 4 <= width) {
            *reinterpret_cast<Anywhere *>(d + k) = out;
        } else {
#pragma unroll
            for (int e = 0; e < 4; e++)
                if (k + e < width) d[k + e] = out[e];
        }
    }
}

// ---------------------------------------------------------------- launches

// Three tiles.  The large one reads each operand least often; the smaller ones fill the chip's 256 compute units (one, two and four blocks
// each) where there are few of it, or where the tokens do not fill its rows.  Binary32 products are bound by the matrix cores, which the
// tiny tile keeps as busy as the others, with more of it in flight and less lost in the last round: us with small and with tiny tiles,
// 300 x 2048 x 30000 with gradients 1450 and 1309, 2000 x 1500 x 5000 1133 and 1048, the loss of 509 x 768 x 30522 200 and 192.
template <typename T, Layout LA, Layout LB>
using Tiny = Tile<T, 64, 64, 4, 1, LA, LB>;
// The tiny one with more of the weight on its way, for one row of tiles, whose blocks all run at a time, three on a compute unit.  Three
// stages in LDS instead of two, us: 32 x 2048 x 50257 56 and 59 to 61, 64 x 2048 x 50257 56 and 59, 64 x 1024 x 50257 24.3 and 23.8.
template <typename T, Layout LA, Layout LB>
using Streamed = Tile<T, 64, 64, 4, 1, LA, LB, 3>;
template <typename T, Layout LA, Layout LB>
using Small = std::conditional_t<sizeof(T) == 2, Tile<T, 128, 128, 2, 2, LA, LB>, Tiny<T, LA, LB>>;
template <typename T, Layout LA, Layout LB>
using Large = std::conditional_t<sizeof(T) == 2, Tile<T, 256, 256, 2, 4, LA, LB>, Tiny<T, LA, LB>>;

int64_t tiles(int64_t rows, int64_t columns, int side) { return ((rows + side - 1) / side) * ((columns + side - 1) / side); }

enum Size { kTiny, kSmall, kLarge };

// Which tile a product of rows x columns takes: the one with the least time, in rounds of the large one, of which the others do 0.91 and
// 0.6 of the work.  split: steps of a summed axis over which a last, partial round may be split (weight_tiles), which costs a pass over
// its parts in a launch of its own (of about three steps' time).  Measured, us with large and with small tiles for the weight's gradient:
// 1500 tokens x 768 x 30522 349 and 332 (1.4 rounds), 2048 x 1024 x 50257 840 and 889 (3.1 rounds, split); for the loss of 2048 x 2048 x
// 50257 353 and 375 (6.2 and 12.3 rounds).
template <typename T>
Size size_of(int64_t rows, int64_t columns, int64_t split = 0)
{
    if (sizeof(T) == 4) return kTiny;
    const auto rounds = [&](int side, int64_t blocks) {
        const int64_t n = tiles(rows, columns, side), rest = n % blocks, most = split / kLeastSteps;
        const int64_t parts = rest && blocks / rest < most ? blocks / rest : most;
        return double(n / blocks) + (!rest ? 0.0 : parts >= 2 ? 1.0 / double(parts) + 0.12 + 3.0 / double(split) : 1.0);
    };
    const double large = rounds(256, kHeadBlocks), small = rounds(128, 2 * kHeadBlocks) * 0.5 / 0.91, tiny = rounds(64, 4 * kHeadBlocks) * 0.25 / 0.6;
    return large <= small && large <= tiny ? kLarge : small <= tiny ? kSmall : kTiny;
}

// d is rounded to 16 bits where the operands have 16.  A target's element, which is most of a row, is near 1 in the units that d is held in and loses
// little; a teacher's entries may be anything.  So the calls of Tempered hold d of few tokens, whose products are bound by reading and writing the
// weights, in two parts of 16 bits (lower: two sections of rows, with the hidden states in both), and that of more bfloat16
// tokens in binary16, against hidden states and weights in binary16 (D; multiplied by a power of two that brings the largest close to that type's
// largest, so that what bfloat16 holds is held to 2^-32 of it).
template <typename T, typename S = Targets, typename D = T>
struct Calls {
    const HeadLayout &l;
    const HeadBuffers &b;
    hipStream_t stream;
    S softmax = S();
    typename S::Picks picks = typename S::Picks();
    int32_t *tokens_of_rows = nullptr;
    bool lower = false;
    bool few_logits = false;                                               // d is formed by what entries() queues
    bool copied = false;                                                   // hidden states are read from their copies, whichever tokens count
    D *hidden_of_products = nullptr, *weight_of_products = nullptr;        // where D is another type
    float *scales = nullptr;                                               // of the hidden states, of the weight's piece: 1 / the power of two
    static constexpr bool kOther = !std::is_same<D, T>::value;
    static constexpr bool kFewOnly = !S::kTargets && std::is_same<D, __bf16>::value;       // d of more tokens is held in binary16
    mutable hipError_t error = hipSuccess;      // of the first launch that was refused

    void launched() const
    {
        const hipError_t e = hipGetLastError();
        if (error == hipSuccess) error = e;
    }

    // Blocks that the chip holds at a time: one of the large tile per compute unit, two of the small one, four of the tiny one.
    template <typename K>
    static constexpr int blocks = K::BM == 256 ? kHeadBlocks : K::BM == 128 ? 2 * kHeadBlocks : 4 * kHeadBlocks;
    template <typename U>
    U *at(size_t offset) const
    {
        return reinterpret_cast<U *>(b.workspace + offset);
    }
    Header *header() const { return at<Header>(0); }
    Hidden<T> hidden() const
    {
        // (whole steps of tokens: the gradient's products sum over them)
        const bool fits = !copied && !l.padded && l.tokens % head_depth(l.dt) == 0;
        return Hidden<T>{fits ? static_cast<const T *>(b.hidden) : nullptr, at<T>(l.hidden), l.tokens};
    }
    // The list, and the first piece of the weight in padded rows where they have to be.
    void list(const float *dloss, const float *lse, float outer = 1.f) const
    {
        const Hidden<T> h = hidden();
        const int64_t n = (l.tokens + 15) / 16, grid = n < 1 ? 1 : n < kHeadBlocks ? n : kHeadBlocks;
        const int64_t columns = l.padded && l.tokens ? l.columns(0) : 0, wanted = (columns + kListThreads / 64 - 1) / (kListThreads / 64);
        const int64_t pads = wanted < 8 * kHeadBlocks ? wanted : 8 * kHeadBlocks;
        list_tokens<T><<<dim3(uint32_t(grid + pads)), kListThreads, 0, stream>>>(
            b.targets, dloss, lse, l.tokens, b.ignore, l.vocab, kTopBits, outer, static_cast<const T *>(b.hidden), l.width, at<T>(l.hidden), l.pitch, int32_t(head_depth(l.dt)), h.own ? 1 : 0, header(),
            Lists{at<int32_t>(l.place), at<int32_t>(l.target), at<float>(l.lse), at<float>(l.factor), tokens_of_rows}, uint32_t(grid),
            Padding<T>{static_cast<const T *>(b.weight), at<T>(l.weight), columns, l.width, l.pitch});
        launched();
    }
    // Rows `first` on of the weight, as the products read them.  (list() has padded the first piece.)
    const T *weight(int64_t first, int64_t columns) const
    {
        const T *w = static_cast<const T *>(b.weight) + first * l.width;
        if (!l.padded) return w;
        if (first > 0) {
            pad_rows<T><<<dim3(uint32_t(columns)), 256, 0, stream>>>(w, l.width, at<T>(l.weight), l.pitch);
            launched();
        }
        return at<T>(l.weight);
    }

    template <typename K>
    void loss_piece(int64_t first, int64_t columns) const
    {
        loss_tiles<K, S><<<dim3(uint32_t(tiles(l.tokens, columns, K::BM))), K::kThreads, 0, stream>>>(
            tokens(), direct() ? Hidden<T>{static_cast<const T *>(b.hidden), nullptr, l.tokens} : hidden(), weight(first, columns), l.pitch,
            first, columns, l.parts, at<float2>(l.stats), at<float>(l.picked), softmax, picks);
        launched();
    }
    void loss_of_few() const
    {
        const uint32_t groups = uint32_t((l.tokens + kFewTokens - 1) / kFewTokens);
        uint32_t more = 0;
        if constexpr (!S::kTargets) more = picks.blocks;
        few_tiles<T, S><<<dim3(uint32_t((l.vocab + kFewColumns - 1) / kFewColumns) * groups + more), 64 * kFewWaves, 0, stream>>>(
            tokens(), static_cast<const T *>(b.hidden), static_cast<const T *>(b.weight), l.width, groups, l.parts, at<float2>(l.stats),
            at<float>(l.picked), softmax, picks);
        launched();
    }
    template <int WAVES>
    void join(int side, float *loss, float *lse) const
    {
        constexpr int kPerBlock = join_tokens<WAVES>;
        join_loss<WAVES><<<dim3(uint32_t((l.tokens + kPerBlock - 1) / kPerBlock)), 64 * WAVES * kPerBlock, 0, stream>>>(
            tokens(), (l.vocab + side - 1) / side, l.parts, at<float2>(l.stats), at<float>(l.picked), loss, lse);
        launched();
    }
    // Tokens of few_tiles: it reads rows that start anywhere, which the tiles need padded, at three times the weight's traffic; a second group of
    // 16 tokens takes the weight again.  us with it and with padding: 16 x 1198 x 50257 bfloat16 31 and 84, 32 x 1198 x 50257 52 and 79, 64 x
    // 1198 x 50257 94 and 83; rows of an odd number of 16-bit elements, whose loads cost more, 1 x 1537 x 50257 75 and 96, 16 x 1537 x 50257
    // 105 and 96, 16 x 1537 x 5000 22 and 27, 48 x 1537 x 5000 36 and 27.
    // Where tiles would leave most of the chip idle it has eight times as many blocks, a quarter of the sums each, and needs no list.  us with it
    // and with tiles: 125 x 519 x 1003 binary32 (32 tiles) 12.7 and 24.5, 256 x 1024 x 1000 bfloat16 (64) 13 and 17, binary32 19 and 30; 256 x
    // 1024 x 2000 bfloat16 (128) 18 and 17, 256 x 1024 x 4000 (252) 28.7 and 18; rows of an odd number of 16-bit elements, 100 x 1537 x 2000 (64),
    // 35 and 27.
    bool few() const
    {
        const bool words = l.width * sizeof(T) % 4 == 0;
        const bool twice = l.padded && words && l.vocab < int64_t(1) << 27;      // (two groups' grid stays under 2^32 threads)
        return l.tokens <= (twice ? 2 * kFewTokens : kFewTokens) || few_of_both();
    }
    // (what few() says of few logits)
    bool few_of_both() const { return l.width * sizeof(T) % 4 == 0 && tiles(l.tokens, l.vocab, 64) <= kFewTiles; }
    bool direct() const { return few() || (l.tokens <= kDirectTokens && !l.padded); }
    Tokens tokens() const
    {
        return Tokens{direct() ? nullptr : header(), at<int32_t>(l.place), at<int32_t>(l.target), b.targets, l.tokens, b.ignore, l.vocab};
    }
    // The parts of all rows' softmax; returns how many columns of the vocabulary a part has.
    int loss_parts() const
    {
        if (direct()) {
            if (few()) loss_of_few();
            else loss_piece<Streamed<T, kSumContiguous, kSumStrips>>(0, l.vocab);
            return few() ? kFewColumns : 64;
        }
        list(nullptr, nullptr);
        // (a weight that needs no padding is walked in one launch)
        const int64_t piece = l.padded ? l.piece : l.vocab;
        const Size size = size_of<T>(l.tokens, piece);
        for (int64_t first = 0; first < l.vocab; first += piece) {
            const int64_t columns = l.vocab - first < piece ? l.vocab - first : piece;
            if (size == kLarge) loss_piece<Large<T, kSumContiguous, kSumStrips>>(first, columns);
            else if (size == kSmall) loss_piece<Small<T, kSumContiguous, kSumStrips>>(first, columns);
            else loss_piece<Tiny<T, kSumContiguous, kSumStrips>>(first, columns);
        }
        return size == kLarge ? 256 : size == kSmall ? 128 : 64;
    }
    hipError_t loss(float *loss, float *lse) const
    {
        const int side = loss_parts();
        if (direct()) join<kJoinWaves>(side, loss, lse);
        else join<1>(side, loss, lse);
        return error;
    }

    template <typename K, typename BESIDE>
    void delta(const T *w, int64_t first, int64_t columns, const BESIDE &beside) const
    {
        const auto go = [&](auto in_two) {
            delta_tiles<K, S, D, decltype(in_two)::value, BESIDE><<<dim3(uint32_t(tiles(l.tokens, columns, K::BM)) + beside.blocks), K::kThreads, 0, stream>>>(
                header(), hidden(), w, l.pitch, first, columns, at<int32_t>(l.target), at<float>(l.lse), at<float>(l.factor), at<D>(l.delta),
                l.piece, softmax, beside);
            launched();
        };
        if constexpr (!S::kTargets && !kOther && sizeof(T) == 2 && K::BM == 64) {
            if (kFewOnly || lower) return go(std::true_type());
        }
        if constexpr (!kFewOnly) go(std::false_type());
    }
    // What the products of d run over: the rows that count, or (lower) two sections of them.
    Header *products() const { return header() + (lower ? 1 : 0); }
    int64_t product_rows() const { return lower ? 2 * lower_rows(l.tokens) : l.tokens; }
    Hidden<D> product_hidden() const
    {
        if constexpr (kOther) return Hidden<D>{nullptr, hidden_of_products, l.tokens};
        else {
            const Hidden<T> h = hidden();
            return Hidden<D>{lower ? nullptr : h.own, h.listed, l.tokens};
        }
    }
    // The tile of dx: its sum over the vocabulary is split where there are few of it, so that any size fills the chip, and each part is written
    // and read again.  The larger tile, then, where it needs few parts.  Whole calls with large and with small tiles, us: 2048 x 1024 x 50257 (32
    // large tiles) 846 and 896, 600 x 2048 x 50257 (24) 629 and 619, 1500 x 768 x 30522 (18) 346 and 344.
    Size sums_size() const
    {
        if (sizeof(T) == 4 || product_rows() <= 64) return kTiny;
        const auto blocks_of = [&](int side, int64_t most) {
            const int64_t n = tiles(product_rows(), l.pitch, side), parts = l.piece / (kLeastSteps * head_depth(l.dt));
            return n * (most / n < 1 ? 1 : most / n < parts ? most / n : parts);
        };
        if (tiles(product_rows(), l.pitch, 256) >= 32 && blocks_of(256, blocks<Large<T, kSumContiguous, kRowContiguous>>) >= 192) return kLarge;
        return blocks_of(128, 2 * kHeadBlocks) >= 384 ? kSmall : kTiny;
    }
    template <typename K>
    void hidden_sums(const D *w, int64_t first, int64_t columns) const
    {
        const int64_t n = tiles(product_rows(), l.pitch, K::BM);
        hidden_tiles<K, kOther><<<dim3(uint32_t(n > blocks<K> ? n : blocks<K>)), K::kThreads, 0, stream>>>(
            products(), at<D>(l.delta), l.piece, w, l.pitch, columns, blocks<K>, first > 0, at<float>(l.sums), kOther ? scales + 1 : nullptr);
        launched();
    }
    // Both products of few tokens that are not listed: the host knows how many tiles have something to do.  (They need no weight_rest: few steps.)
    template <typename KH, typename KW>
    void both_products(const T *w, int64_t first, int64_t columns, T *dweight) const
    {
        const uint32_t tiles_h = uint32_t(tiles(product_rows(), l.pitch, KH::BM)), of_hidden = tiles_h * parts_of(tiles_h, up(l.piece, KH::kDepth), blocks<KH>);
        const Rounds r = rounds_of(uint32_t(tiles(columns, l.width, KW::BM)), up(product_rows(), KW::kDepth), blocks<KW>);
        both_tiles<KH, KW><<<dim3(of_hidden + r.whole + r.rest * r.parts), KH::kThreads, 0, stream>>>(
            of_hidden, products(), at<T>(l.delta), l.piece, w, l.pitch, columns, blocks<KH>, first > 0, at<float>(l.sums), product_hidden(), l.width,
            dweight + first * l.width, at<float>(l.spare));
        launched();
    }
    template <typename K>
    void rounded(T *dhidden) const
    {
        const auto go = [&](auto in_two) {
            round_hidden<T, decltype(in_two)::value><<<dim3(uint32_t(l.tokens)), 256, 0, stream>>>(
                products(), at<int32_t>(l.place), at<float>(l.sums), l.pitch, l.width, K::BM, int32_t((l.piece + K::kDepth - 1) / K::kDepth), blocks<K>,
                dhidden);
            launched();
        };
        if constexpr (!S::kTargets && !kOther && sizeof(T) == 2) {
            if (kFewOnly || lower) return go(std::true_type());
        }
        if constexpr (!kFewOnly) go(std::false_type());
    }
    template <typename K>
    void weight_rows(int64_t first, int64_t columns, T *dweight) const
    {
        const int64_t n = tiles(columns, l.width, K::BM), rest = n % blocks<K>;
        // (whether the rest is split depends on how many tokens count, too)
        weight_tiles<K, T, kOther><<<dim3(uint32_t(n - rest + (rest ? blocks<K> : 0))), K::kThreads, 0, stream>>>(
            products(), at<D>(l.delta), l.piece, product_hidden(), l.pitch, columns, l.width, blocks<K>, dweight + first * l.width,
            at<float>(l.spare), scales);
        launched();
        if (!rest || 2 * rest > blocks<K> || (product_rows() + K::kDepth - 1) / K::kDepth < 2 * kLeastSteps) return;
        if constexpr (!kFewOnly) {                       // (few steps are not split)
            weight_rest<K, T, kOther><<<dim3(uint32_t(rest * (K::BM / 16))), 256, 0, stream>>>(products(), columns, l.width, blocks<K>,
                                                                                            dweight + first * l.width, at<float>(l.spare), scales);
            launched();
        }
    }
    static constexpr int kTopBits = std::is_same<D, _Float16>::value ? 14 : std::is_same<D, __bf16>::value ? kLift : 0;
    // listed(): queues the list of tokens and what the products' hidden states need; entries(w, first, columns): what d of a piece lacks, and what the
    // products' weights need.
    // beside(first, columns): what d's launch does besides.
    template <class Listed, class Beside, class Entries>
    hipError_t gradient(T *dhidden, T *dweight, Listed listed, Beside beside, Entries entries) const
    {
        listed();
        const Size sums = sums_size();
        for (int64_t k = 0; k < l.pieces; k++) {
            const int64_t first = k * l.piece, columns = l.columns(k);
            const T *w = l.tokens ? weight(first, columns) : nullptr;
            if (l.tokens) {
                const Size size = kFewOnly || lower ? kTiny : size_of<T>(l.tokens, columns);
                if (few_logits) {
                } else if (size == kLarge) delta<Large<T, kSumContiguous, kSumStrips>>(w, first, columns, beside(first, columns));
                else if (size == kSmall) delta<Small<T, kSumContiguous, kSumStrips>>(w, first, columns, beside(first, columns));
                else delta<Tiny<T, kSumContiguous, kSumStrips>>(w, first, columns, beside(first, columns));
                entries(w, first, columns);
                const D *of;
                if constexpr (kOther) of = weight_of_products;
                else of = w;
                if constexpr (!S::kTargets && !kOther) {
                    // (neither product's tiles fill the chip)
                    if (copied && sums == kTiny && tiles(columns, l.width, 64) <= blocks<Tiny<D, kRowContiguous, kRowContiguous>>) {
                        both_products<Tiny<D, kSumContiguous, kRowContiguous>, Tiny<D, kRowContiguous, kRowContiguous>>(of, first, columns, dweight);
                        continue;
                    }
                }
                if (sums == kLarge) hidden_sums<Large<D, kSumContiguous, kRowContiguous>>(of, first, columns);
                else if (sums == kSmall) hidden_sums<Small<D, kSumContiguous, kRowContiguous>>(of, first, columns);
                else hidden_sums<Tiny<D, kSumContiguous, kRowContiguous>>(of, first, columns);
            }
            const Size size = size_of<T>(columns, l.width, (product_rows() + head_depth(l.dt) - 1) / head_depth(l.dt));
            if (size == kLarge) weight_rows<Large<D, kRowContiguous, kRowContiguous>>(first, columns, dweight);
            else if (size == kSmall) weight_rows<Small<D, kRowContiguous, kRowContiguous>>(first, columns, dweight);
            else weight_rows<Tiny<D, kRowContiguous, kRowContiguous>>(first, columns, dweight);
        }
        if (!l.tokens) return error;
        if (sums == kLarge) rounded<Large<D, kSumContiguous, kRowContiguous>>(dhidden);
        else if (sums == kSmall) rounded<Small<D, kSumContiguous, kRowContiguous>>(dhidden);
        else rounded<Tiny<D, kSumContiguous, kRowContiguous>>(dhidden);
        return error;
    }
};

}  // namespace
}  // namespace cgx
