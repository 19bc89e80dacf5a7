// The head's kernels and their launches: softmax cross entropy over a vocabulary without its logits, and its gradient.
//
// With x the hidden states of the N tokens that count, W the weight, z = x W^T:
//   loss call      z tile by tile; each tile leaves its rows' largest logit and sum of exp(z - largest), which a last kernel joins
//   gradient call  for each piece of the vocabulary: z again, d = dloss (exp(z - lse) - [v = target]) into the workspace,
//                  dx += d W, dW = d^T x
// 2 N V H operations for the loss, 2 N V H + 4 N V H for the gradient, against (N + V) H elements read: above some hundred
// tokens everything is bound by the matrix cores, below by reading W.
#include "cgx_head.h"

#include "cgx_head_gemm.h"

namespace cgx {
namespace {

using namespace gemm;

constexpr float kLog2e = 1.44269504088896340736f;

struct Header {
    int32_t count;           // tokens that count
    float unscale;           // a power of two: what the products of d are multiplied by
};

// 2^LIFT exp(x) of a logit's distance from the log-sum-exp or from a part's largest logit.  The binary32 calls take the library
// function (1 ulp): their results are held to binary32 accuracy; for 16-bit types the hardware's exp2 is far below their own rounding.
template <typename T, int LIFT = 0>
__device__ __forceinline__ float exp_of(float x)
{
    if constexpr (sizeof(T) == 4) return expf(x);
    else return __builtin_amdgcn_exp2f(__builtin_fmaf(x, kLog2e, float(LIFT)));
}

// The hardware's exp2 gives 0 below 2^-126; d of 16-bit types is formed from probabilities lifted by this much, which keeps those
// down to 2^-150, and its scale takes the lift out again.
constexpr int kLift = 24;
template <typename T>
constexpr int lift_of = sizeof(T) == 2 ? kLift : 0;

// ---------------------------------------------------------------- which tokens count

// One block lists the tokens that count, in order, with their targets and factors.  A token takes part if its target is not
// `ignore` and (gradient) its factor is not 0; the products then run over that list alone.
// Each thread takes a run of neighbouring tokens; a prefix sum over the threads' counts gives the places.
constexpr int kListThreads = 1024;

__global__ __launch_bounds__(kListThreads) void list_tokens(const int64_t *__restrict__ targets, const float *__restrict__ dloss,
                                                            const float *__restrict__ lse_in, int64_t tokens, int64_t rows,
                                                            int64_t ignore, int64_t vocab, int32_t top_bits, Header *header,
                                                            int32_t *__restrict__ index, int32_t *__restrict__ place,
                                                            int32_t *__restrict__ target, float *__restrict__ lse,
                                                            float *__restrict__ factor)
{
    __shared__ int32_t counts[kListThreads / 64];
    __shared__ float tops[kListThreads / 64];
    const int tid = int(threadIdx.x), lane = tid & 63, wave = tid >> 6;
    const int64_t each = (tokens + kListThreads - 1) / kListThreads, first = int64_t(tid) * each;
    const int64_t end = first + each < tokens ? first + each : tokens;
    int32_t mine = 0;
    float top = 0.f;
    for (int64_t t = first; t < end; t++) {
        const float g = dloss ? dloss[t] : 1.f;
        if (targets[t] == ignore || g == 0.f) continue;
        mine++;
        top = fmaxf(top, fabsf(g));
    }
    int32_t before = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int32_t other = __shfl_up(before, d, 64);
        if (lane >= d) before += other;
        top = fmaxf(top, __shfl_xor(top, d, 64));
    }
    if (lane == 63) counts[wave] = before;
    if (lane == 0) tops[wave] = top;
    __syncthreads();
    int32_t count = 0;
    before -= mine;
    for (int w = 0; w < kListThreads / 64; w++) {
        before += w < wave ? counts[w] : 0;
        count += counts[w];
        top = fmaxf(top, tops[w]);
    }
    // d is held under a power of two that moves the largest factor to [2^top_bits, 2^(top_bits + 1)): in binary16, with 14,
    // probabilities down to 1e-9 stay normal numbers and nothing overflows, whatever the loss scale
    int shift = 0;
    if (top_bits && top > 0.f && top < __builtin_inff()) {
        shift = top_bits - ilogbf(top);
        shift = shift > 120 ? 120 : shift < -120 ? -120 : shift;
    }
    const float scale = ldexpf(1.f, shift - (top_bits ? kLift : 0));
    if (tid == 0) *header = Header{count, ldexpf(1.f, -shift)};
    for (int64_t t = first; t < end; t++) {
        const float g = dloss ? dloss[t] : 1.f;
        const int64_t v = targets[t];
        if (v == ignore || g == 0.f) {
            place[t] = -1;
            continue;
        }
        const bool outside = v < 0 || v >= vocab;
        index[before] = int32_t(t);
        place[t] = before;
        target[before] = outside ? -1 : int32_t(v);
        if (dloss) {
            lse[before] = lse_in[t];
            factor[before] = outside ? __builtin_nanf("") : g * scale;
        }
        before++;
    }
}

// ---------------------------------------------------------------- rows into place

// A block per row: dst[row][0 .. pitch) = src[index ? index[row] : row][0 .. width), then zeros.  With a header, rows past the
// count are zeros up to a whole step of the products' summed axis, and not written beyond.
template <typename T>
__global__ __launch_bounds__(256) void copy_rows(const T *__restrict__ src, int64_t width, T *__restrict__ dst, int64_t pitch,
                                                 const Header *header, const int32_t *__restrict__ index, int32_t depth, int32_t in_place)
{
    constexpr int kPer = 16 / int(sizeof(T));
    typedef uint32_t Vec __attribute__((ext_vector_type(4)));
    int64_t row = blockIdx.x, from = row;
    if (header) {
        const int64_t count = header->count;
        // the products read the hidden states themselves, see hidden_of
        if (in_place && count == gridDim.x) return;
        if (row >= (count + depth - 1) / depth * depth) return;
        from = row < count ? index[row] : -1;
    }
    const T *s = src + from * width;
    T *d = dst + row * pitch;
    if (from < 0) {
        for (int64_t k = int64_t(threadIdx.x) * kPer; k < pitch; k += 256 * kPer) *reinterpret_cast<Vec *>(d + k) = Vec{0, 0, 0, 0};
    } else if (width % kPer == 0) {
        for (int64_t k = int64_t(threadIdx.x) * kPer; k < pitch; k += 256 * kPer)
            *reinterpret_cast<Vec *>(d + k) = k < width ? *reinterpret_cast<const Vec *>(s + k) : Vec{0, 0, 0, 0};
    } else {
        for (int64_t k = int64_t(threadIdx.x); k < pitch; k += 256) d[k] = k < width ? s[k] : T(0.f);
    }
}

// The hidden states that the products read: the caller's where every token counts and their rows fit the tiles as they are.
template <typename T>
struct Hidden {
    const T *own;            // or null: never
    const T *listed;
    int64_t tokens;
    __device__ __forceinline__ const T *of(int64_t count) const { return own && count == tokens ? own : listed; }
};

// ---------------------------------------------------------------- logits

__device__ __forceinline__ uint32_t up(int64_t v, int to) { return uint32_t((v + to - 1) / to); }

template <typename K>
using Lds = unsigned char[K::kLds];

// Logits of a tile, and what its rows add to their softmax: the largest logit, the sum of exp(logit - it).
template <typename K>
__global__ __launch_bounds__(K::kThreads, 2) void loss_tiles(const Header *header, Hidden<typename K::T> hidden, const typename K::T *weight,
                                                          int64_t pitch, int64_t first, int64_t columns, int64_t rows,
                                                          const int32_t *__restrict__ target, float2 *__restrict__ stats,
                                                          float *__restrict__ picked)
{
    using T = typename K::T;
    __shared__ __align__(256) Lds<K> lds;
    const int64_t count = header->count;
    int tm, tn;
    if (!tile_of_block(blockIdx.x, up(count, K::BM), up(columns, K::BN), tm, tn)) return;
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
    const int64_t c0 = n0 + tile.wn + 4 * g;
    const bool whole = n0 + K::BN <= columns;
#pragma unroll
    for (int i = 0; i < K::TM; i++) {
        const int m = tile.wm + 16 * i + r;
        const int64_t row = m0 + m;
        if (row < count) {
            const int64_t d = int64_t(target[row]) - first - c0;
            if (d >= 0 && d < 16 * K::TN && (d & 15) < 4) {
#pragma unroll
                for (int j = 0; j < K::TN; j++)
#pragma unroll
                    for (int e = 0; e < 4; e++)
                        if (d == 16 * j + e) picked[row] = tile.acc[i][j][e];
            }
        }
        float top = -__builtin_inff();
#pragma unroll
        for (int j = 0; j < K::TN; j++)
#pragma unroll
            for (int e = 0; e < 4; e++) {
                if (!whole && c0 + 16 * j + e >= columns) tile.acc[i][j][e] = -__builtin_inff();
                top = fmaxf(top, tile.acc[i][j][e]);
            }
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float from = top == -__builtin_inff() ? 0.f : top;
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < K::TN; j++)
#pragma unroll
            for (int e = 0; e < 4; e++) sum += exp_of<T>(tile.acc[i][j][e] - from);
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
        stats[((first + n0) / K::BN) * rows + m0 + m] = float2{top, sum};
    }
}

// Joins the parts of every token's softmax: 64 rows per block, four threads each.
__global__ __launch_bounds__(256) void join_loss(int64_t tokens, int64_t rows, int64_t parts, const int32_t *__restrict__ place,
                                                 const int32_t *__restrict__ target, const float2 *__restrict__ stats,
                                                 const float *__restrict__ picked, float *__restrict__ loss, float *__restrict__ lse)
{
    __shared__ float2 quarter[4][64];
    const int at = int(threadIdx.x) & 63, q = int(threadIdx.x) >> 6;
    const int64_t token = int64_t(blockIdx.x) * 64 + at;
    const int32_t row = token < tokens ? place[token] : -1;
    float top = -__builtin_inff(), sum = 0.f;
    if (row >= 0) {
        for (int64_t p = q; p < parts; p += 4) top = fmaxf(top, stats[p * rows + row].x);
        const float from = top == -__builtin_inff() ? 0.f : top;
        for (int64_t p = q; p < parts; p += 4) {
            const float2 s = stats[p * rows + row];
            sum += s.y * expf(s.x - from);
        }
    }
    quarter[q][at] = float2{top, sum};
    __syncthreads();
    if (q != 0 || token >= tokens) return;
    if (row < 0) {
        loss[token] = 0.f;
        lse[token] = 0.f;
        return;
    }
#pragma unroll
    for (int k = 1; k < 4; k++) top = fmaxf(top, quarter[k][at].x);
    const float from = top == -__builtin_inff() ? 0.f : top;
    sum = 0.f;
#pragma unroll
    for (int k = 0; k < 4; k++) sum += quarter[k][at].y * expf(quarter[k][at].x - from);
    const float all = from + logf(sum);
    lse[token] = all;
    loss[token] = target[row] < 0 ? __builtin_nanf("") : all - picked[row];
}

// ---------------------------------------------------------------- gradient

// d of a tile of a piece: logits as above, then dloss (exp(z - lse) - [v = target]) under the scale, in the operands' type.
// Every element of the piece's whole tiles is written; those of no token or no column are zeros.
template <typename K>
__global__ __launch_bounds__(K::kThreads, 2) void delta_tiles(const Header *header, Hidden<typename K::T> hidden, const typename K::T *weight,
                                                           int64_t pitch, int64_t first, int64_t columns,
                                                           const int32_t *__restrict__ target, const float *__restrict__ lse,
                                                           const float *__restrict__ factor, typename K::T *__restrict__ delta, int64_t piece)
{
    using T = typename K::T;
    typedef T Four __attribute__((ext_vector_type(4)));
    __shared__ __align__(256) Lds<K> lds;
    const int64_t count = header->count;
    int tm, tn;
    if (!tile_of_block(blockIdx.x, up(count, K::BM), up(columns, K::BN), tm, tn)) return;
    const int64_t m0 = int64_t(tm) * K::BM, n0 = int64_t(tn) * K::BN;
    K tile;
    typename K::A a;
    typename K::B b;
    a.start(hidden.of(count), pitch, m0, count - m0, 0, int(threadIdx.x));
    b.start(weight, pitch, n0, columns - n0, 0, int(threadIdx.x));
    tile.run(a, b, int(pitch / K::kDepth), K::kDepth, lds);

    const int g = tile.lane >> 4, r = tile.lane & 15;
    const int64_t c0 = n0 + tile.wn + 4 * g;
    const bool whole = n0 + K::BN <= columns;
#pragma unroll
    for (int i = 0; i < K::TM; i++) {
        const int64_t row = m0 + tile.wm + 16 * i + r;
        const bool counts = row < count;
        const float base = counts ? lse[row] : 0.f, f = counts ? factor[row] : 0.f;
        const int64_t hit = counts ? int64_t(target[row]) - first - c0 : -1;
#pragma unroll
        for (int j = 0; j < K::TN; j++) {
            Four out;
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const float p = exp_of<T, lift_of<T>>(tile.acc[i][j][e] - base);
                const float v = (hit == 16 * j + e ? p - float(1 << lift_of<T>) : p) * f;
                out[e] = T(counts && (whole || c0 + 16 * j + e < columns) ? v : 0.f);
            }
            *reinterpret_cast<Four *>(delta + row * piece + c0 + 16 * j) = out;
        }
    }
}

// dx += d W over a piece.  accumulate: not the first piece.
template <typename K>
__global__ __launch_bounds__(K::kThreads, 2) void hidden_tiles(const Header *header, const typename K::T *delta, int64_t piece,
                                                            const typename K::T *weight, int64_t pitch, int64_t columns, int32_t accumulate,
                                                            float *__restrict__ sums)
{
    __shared__ __align__(256) Lds<K> lds;
    const int64_t count = header->count;
    int tm, tn;
    if (!tile_of_block(blockIdx.x, up(count, K::BM), up(pitch, K::BN), tm, tn)) return;
    const int64_t m0 = int64_t(tm) * K::BM, n0 = int64_t(tn) * K::BN;
    K tile;
    typename K::A a;
    typename K::B b;
    a.start(delta, piece, m0, count - m0, 0, int(threadIdx.x));
    b.start(weight, pitch, n0, pitch - n0, 0, int(threadIdx.x));
    const int steps = int(up(columns, K::kDepth));
    tile.run(a, b, steps, int(columns - int64_t(steps - 1) * K::kDepth), lds);
    const int g = tile.lane >> 4, r = tile.lane & 15;
#pragma unroll
    for (int i = 0; i < K::TM; i++) {
        const int64_t row = m0 + tile.wm + 16 * i + r;
        if (row >= count) continue;
#pragma unroll
        for (int j = 0; j < K::TN; j++) {
            const int64_t column = n0 + tile.wn + 16 * j + 4 * g;
            if (column >= pitch) continue;
            f32x4 *p = reinterpret_cast<f32x4 *>(sums + row * pitch + column);
            *p = accumulate ? *p + tile.acc[i][j] : tile.acc[i][j];
        }
    }
}

// dW = d^T x for the rows of a piece.
template <typename K>
__global__ __launch_bounds__(K::kThreads, 2) void weight_tiles(const Header *header, const typename K::T *delta, int64_t piece,
                                                            Hidden<typename K::T> hidden, int64_t pitch, int64_t columns, int64_t width,
                                                            typename K::T *__restrict__ dweight)
{
    using T = typename K::T;
    typedef T Four __attribute__((ext_vector_type(4)));
    __shared__ __align__(256) Lds<K> lds;
    const int64_t count = header->count;
    int tm, tn;
    if (!tile_of_block(blockIdx.x, up(columns, K::BM), up(width, K::BN), tm, tn)) return;
    const int64_t m0 = int64_t(tm) * K::BM, n0 = int64_t(tn) * K::BN;
    const float unscale = header->unscale;
    K tile;
    typename K::A a;
    typename K::B b;
    a.start(delta, piece, m0, piece - m0, 0, int(threadIdx.x));
    b.start(hidden.of(count), pitch, n0, pitch - n0, 0, int(threadIdx.x));
    tile.run(a, b, int(up(count, K::kDepth)), K::kDepth, lds);
    const int g = tile.lane >> 4, r = tile.lane & 15;
    const bool fours = width % 4 == 0;
#pragma unroll
    for (int i = 0; i < K::TM; i++) {
        const int64_t row = m0 + tile.wm + 16 * i + r;
        if (row >= columns) continue;
#pragma unroll
        for (int j = 0; j < K::TN; j++) {
            const int64_t column = n0 + tile.wn + 16 * j + 4 * g;
            if (column >= width) continue;
            T *p = dweight + row * width + column;
            Four out;
#pragma unroll
            for (int e = 0; e < 4; e++) out[e] = T(tile.acc[i][j][e] * unscale);
            if (fours) {
                *reinterpret_cast<Four *>(p) = out;
            } else {
#pragma unroll
                for (int e = 0; e < 4; e++)
                    if (column + e < width) p[e] = out[e];
            }
        }
    }
}

// dhidden from the sums; a block per token.
template <typename T>
__global__ __launch_bounds__(256) void round_hidden(const Header *header, const int32_t *__restrict__ place, const float *__restrict__ sums,
                                                    int64_t pitch, int64_t width, T *__restrict__ dhidden)
{
    typedef T Four __attribute__((ext_vector_type(4)));
    const int64_t token = blockIdx.x;
    const int32_t row = place[token];
    const float unscale = header->unscale;
    const float *s = sums + int64_t(row < 0 ? 0 : row) * pitch;
    T *d = dhidden + token * width;
    if (width % 4 == 0) {
        for (int64_t k = int64_t(threadIdx.x) * 4; k < width; k += 1024) {
            const f32x4 v = row < 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : *reinterpret_cast<const f32x4 *>(s + k);
            Four out;
#pragma unroll
            for (int e = 0; e < 4; e++) out[e] = T(v[e] * unscale);
            *reinterpret_cast<Four *>(d + k) = out;
        }
    } else {
        for (int64_t k = int64_t(threadIdx.x); k < width; k += 256) d[k] = T(row < 0 ? 0.f : s[k] * unscale);
    }
}

// ---------------------------------------------------------------- launches

template <typename T, Layout LA, Layout LB>
using Small = Tile<T, 128, 128, 2, 2, LA, LB>;
template <typename T, Layout LA, Layout LB>
using Large = std::conditional_t<sizeof(T) == 2, Tile<T, 256, 256, 2, 4, LA, LB>, Small<T, LA, LB>>;

int64_t tiles(int64_t rows, int64_t columns, int side) { return ((rows + side - 1) / side) * ((columns + side - 1) / side); }

// The large tile reads each operand half as often, the small one fills the chip's 256 compute units from a quarter of the size.
template <typename T>
bool large(int64_t rows, int64_t columns)
{
    return sizeof(T) == 2 && tiles(rows, columns, 256) >= 192;
}

template <typename T>
struct Calls {
    const HeadLayout &l;
    const HeadBuffers &b;
    hipStream_t stream;
    mutable hipError_t error = hipSuccess;      // of the first launch that was refused

    void launched() const
    {
        const hipError_t e = hipGetLastError();
        if (error == hipSuccess) error = e;
    }

    template <typename U>
    U *at(size_t offset) const
    {
        return reinterpret_cast<U *>(b.workspace + offset);
    }
    Header *header() const { return at<Header>(0); }
    Hidden<T> hidden() const
    {
        // (whole steps of tokens: the gradient's products sum over them)
        const bool fits = !l.padded && l.tokens % head_depth(l.dt) == 0;
        return Hidden<T>{fits ? static_cast<const T *>(b.hidden) : nullptr, at<T>(l.hidden), l.tokens};
    }
    void list(const float *dloss, const float *lse) const
    {
        list_tokens<<<1, kListThreads, 0, stream>>>(b.targets, dloss, lse, l.tokens, l.rows, b.ignore, l.vocab,
                                                    l.dt == CGX_F16 ? 14 : l.dt == CGX_BF16 ? kLift : 0, header(), at<int32_t>(l.index), at<int32_t>(l.place),
                                                    at<int32_t>(l.target), at<float>(l.lse), at<float>(l.factor));
        launched();
        const Hidden<T> h = hidden();
        const int64_t depth = head_depth(l.dt), rows = (l.tokens + depth - 1) / depth * depth;
        if (rows) {
            copy_rows<T><<<dim3(uint32_t(rows)), 256, 0, stream>>>(static_cast<const T *>(b.hidden), l.width, at<T>(l.hidden), l.pitch, header(),
                                                                at<int32_t>(l.index), int32_t(depth), h.own ? 1 : 0);
            launched();
        }
    }
    // Rows `first` on of the weight, as the products read them.
    const T *weight(int64_t first, int64_t columns) const
    {
        const T *w = static_cast<const T *>(b.weight) + first * l.width;
        if (!l.padded) return w;
        copy_rows<T><<<dim3(uint32_t(columns)), 256, 0, stream>>>(w, l.width, at<T>(l.weight), l.pitch, nullptr, nullptr, 0, 0);
        launched();
        return at<T>(l.weight);
    }

    template <typename K>
    void loss_piece(int64_t first, int64_t columns) const
    {
        loss_tiles<K><<<dim3(uint32_t(tiles(l.tokens, columns, K::BM))), K::kThreads, 0, stream>>>(
            header(), hidden(), weight(first, columns), l.pitch, first, columns, l.rows, at<int32_t>(l.target), at<float2>(l.stats),
            at<float>(l.picked));
        launched();
    }
    hipError_t loss(float *loss, float *lse) const
    {
        list(nullptr, nullptr);
        // (a weight that needs no padding is walked in one launch)
        const int64_t piece = l.padded ? l.piece : l.vocab;
        const bool big = large<T>(l.tokens, piece);
        for (int64_t first = 0; first < l.vocab; first += piece) {
            const int64_t columns = l.vocab - first < piece ? l.vocab - first : piece;
            if (big) loss_piece<Large<T, kSumContiguous, kSumContiguous>>(first, columns);
            else loss_piece<Small<T, kSumContiguous, kSumContiguous>>(first, columns);
        }
        const int side = big ? 256 : 128;
        join_loss<<<dim3(uint32_t((l.tokens + 63) / 64)), 256, 0, stream>>>(l.tokens, l.rows, (l.vocab + side - 1) / side,
                                                                        at<int32_t>(l.place), at<int32_t>(l.target), at<float2>(l.stats),
                                                                        at<float>(l.picked), loss, lse);
        launched();
        return error;
    }

    template <typename K>
    void delta(const T *w, int64_t first, int64_t columns) const
    {
        delta_tiles<K><<<dim3(uint32_t(tiles(l.tokens, columns, K::BM))), K::kThreads, 0, stream>>>(
            header(), hidden(), w, l.pitch, first, columns, at<int32_t>(l.target), at<float>(l.lse), at<float>(l.factor), at<T>(l.delta),
            l.piece);
        launched();
    }
    template <typename K>
    void hidden_sums(const T *w, int64_t first, int64_t columns) const
    {
        hidden_tiles<K><<<dim3(uint32_t(tiles(l.tokens, l.pitch, K::BM))), K::kThreads, 0, stream>>>(
            header(), at<T>(l.delta), l.piece, w, l.pitch, columns, first > 0, at<float>(l.sums));
        launched();
    }
    template <typename K>
    void weight_rows(int64_t first, int64_t columns, T *dweight) const
    {
        weight_tiles<K><<<dim3(uint32_t(tiles(columns, l.width, K::BM))), K::kThreads, 0, stream>>>(
            header(), at<T>(l.delta), l.piece, hidden(), l.pitch, columns, l.width, dweight + first * l.width);
        launched();
    }
    hipError_t gradient(const float *lse, const float *dloss, T *dhidden, T *dweight) const
    {
        list(dloss, lse);
        for (int64_t k = 0; k < l.pieces; k++) {
            const int64_t first = k * l.piece, columns = l.columns(k);
            const T *w = l.tokens ? weight(first, columns) : nullptr;
            if (l.tokens) {
                if (large<T>(l.tokens, columns)) delta<Large<T, kSumContiguous, kSumContiguous>>(w, first, columns);
                else delta<Small<T, kSumContiguous, kSumContiguous>>(w, first, columns);
                if (large<T>(l.tokens, l.pitch)) hidden_sums<Large<T, kSumContiguous, kRowContiguous>>(w, first, columns);
                else hidden_sums<Small<T, kSumContiguous, kRowContiguous>>(w, first, columns);
            }
            if (large<T>(columns, l.width)) weight_rows<Large<T, kRowContiguous, kRowContiguous>>(first, columns, dweight);
            else weight_rows<Small<T, kRowContiguous, kRowContiguous>>(first, columns, dweight);
        }
        if (l.tokens) {
            round_hidden<T><<<dim3(uint32_t(l.tokens)), 256, 0, stream>>>(header(), at<int32_t>(l.place), at<float>(l.sums), l.pitch, l.width,
                                                                       dhidden);
            launched();
        }
        return error;
    }
};

}  // namespace

int launch_head_loss(const HeadLayout &l, const HeadBuffers &b, float *loss, float *lse, void *stream)
{
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (l.tokens == 0) return hipSuccess;
    if (l.dt == CGX_F32) return Calls<float>{l, b, s}.loss(loss, lse);
    if (l.dt == CGX_F16) return Calls<_Float16>{l, b, s}.loss(loss, lse);
    return Calls<__bf16>{l, b, s}.loss(loss, lse);
}

int launch_head_loss_grad(const HeadLayout &l, const HeadBuffers &b, const float *lse, const float *dloss, void *dhidden, void *dweight,
                          void *stream)
{
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (l.dt == CGX_F32) return Calls<float>{l, b, s}.gradient(lse, dloss, static_cast<float *>(dhidden), static_cast<float *>(dweight));
    if (l.dt == CGX_F16) return Calls<_Float16>{l, b, s}.gradient(lse, dloss, static_cast<_Float16 *>(dhidden), static_cast<_Float16 *>(dweight));
    return Calls<__bf16>{l, b, s}.gradient(lse, dloss, static_cast<__bf16 *>(dhidden), static_cast<__bf16 *>(dweight));
}

}  // namespace cgx
