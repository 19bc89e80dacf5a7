// Distillation through the head from a teacher's largest logits: the Kullback-Leibler divergence of the student's softmax over the whole
// vocabulary from the teacher's over its entries, and its gradients, without the student's logits.
//
// With z the student's logits, T the temperature, q = softmax(teacher / T) over a token's entries and lse = log sum_v exp(z_v / T):
//   loss = sum_k q_k (log q_k + lse - z[id_k] / T),   d_v = dloss / T (exp(z_v / T - lse) - sum_{k: id_k = v} q_k)
// The products are those of the head's loss (cgx_head_kernels.h): its tiles give lse, and d but for the teacher's entries, of which there are a few
// per token.
#include "cgx_distill.h"

#include "cgx_head_kernels.h"

namespace cgx {
namespace {

// What the head's list reads as targets.
constexpr int64_t kTakesPart = 0, kWrong = -1, kNoPart = -2;

struct Teacher {
    const int64_t *ids;
    const void *logits;
    int32_t entries, dt;
    int64_t ignore, vocab;
    float inverse;           // 1 / temperature
    __device__ __forceinline__ float logit(int64_t at) const
    {
        if (dt == CGX_F32) return static_cast<const float *>(logits)[at];
        if (dt == CGX_F16) return float(static_cast<const _Float16 *>(logits)[at]);
        return float(static_cast<const __bf16 *>(logits)[at]);
    }
};

// A token's entries: the largest logit (over the temperature) and the sum of exponentials from it, in every lane of a wave.
struct TeacherRow {
    float top, sum;
    bool wrong;              // an id outside the vocabulary, or a logit that is NaN or +infinity
    __device__ __forceinline__ bool takes_part() const { return wrong || sum > 0.f; }
    __device__ __forceinline__ float share(float scaled) const { return expf(scaled - top) / sum; }
};
__device__ __forceinline__ TeacherRow teacher_row(const Teacher &t, int64_t token, int lane)
{
    TeacherRow r{-__builtin_inff(), 0.f, false};
    const int64_t first = token * t.entries;
    bool wrong = false;
    // (one pass over the entries, each lane with a maximum of its own: the loads are what takes time)
    for (int k = lane; k < t.entries; k += 64) {
        const int64_t id = t.ids[first + k];
        const float x = t.logit(first + k) * t.inverse;
        if (id == t.ignore) continue;
        wrong |= id < 0 || id >= t.vocab || !(x < __builtin_inff());
        const float top = fmaxf(r.top, x);
        if (top == -__builtin_inff()) continue;
        r.sum = r.sum * expf(r.top - top) + expf(x - top);
        r.top = top;
    }
    float top = r.top;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
    r.wrong = __ballot(wrong) != 0;
    r.sum = top == -__builtin_inff() ? 0.f : r.sum * expf(r.top - top);
    r.top = top;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) r.sum += __shfl_xor(r.sum, d, 64);
    return r;
}

// What the kernels after it need of a teacher's rows, a wave per token: which tokens take part; their entries sorted by id; and, for the loss, where
// those of every 64 columns begin, for the gradient, their shares.  M: entries, rounded up to a power of two.  8192 tokens of 64 entries 15 us for the
// loss of 50257 columns (13 MB of strips), 12 for the gradient; 4096 of 128 16 and 12: loads, 21 or 28 dependent steps of the sort in LDS, stores.
constexpr int kRowWaves = 4;
template <int M>
struct RowShared {
    uint64_t key[M];         // id, then place
    float share[M];
};

// In ascending order, by one wave.  (LDS accesses of a wave are in order; the compiler is told not to move them.)
__device__ __forceinline__ void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}
template <int M>
__device__ __forceinline__ void sort_keys(uint64_t *key, int lane)
{
    for (int run = 2; run <= M; run *= 2)
        for (int apart = run / 2; apart > 0; apart /= 2) {
            wave_fence();
            for (int p = lane; p < M / 2; p += 64) {
                const int low = 2 * apart * (p / apart) + p % apart, high = low + apart;
                const uint64_t a = key[low], b = key[high];
                const bool rising = (low & run) == 0;
                if ((a > b) == rising) {
                    key[low] = b;
                    key[high] = a;
                }
            }
        }
    wave_fence();
}

template <int M, bool GRAD>
__device__ __forceinline__ TeacherRow row_entries(const Teacher &teacher, int64_t token, int lane, RowShared<M> &s, Entry *__restrict__ entries,
                                                  float *__restrict__ shares, uint16_t *__restrict__ strips, int64_t pitch)
{
    typedef uint32_t Four __attribute__((ext_vector_type(4)));
    const TeacherRow r = teacher_row(teacher, token, lane);
    const int64_t first = token * teacher.entries;
    uint16_t *const row = strips + token * pitch;
    if (!GRAD && strips)                                 // (rows of strips are whole pieces of 16 bytes)
        for (int64_t strip = lane * 8; strip < pitch; strip += 512) *reinterpret_cast<Four *>(row + strip) = Four(0u);
    if (!r.takes_part()) return r;
    constexpr uint64_t kNone = ~uint64_t(0);
    for (int k = lane; k < M; k += 64) {
        uint64_t key = kNone;
        if (k < teacher.entries) {
            const int64_t id = teacher.ids[first + k];
            if (id != teacher.ignore && id >= 0 && id < teacher.vocab) key = uint64_t(id) << kStripBits | uint64_t(k);
            if (GRAD) s.share[k] = key == kNone ? 0.f : r.share(teacher.logit(first + k) * teacher.inverse);
        }
        s.key[k] = key;
    }
    sort_keys<M>(s.key, lane);
    const auto id_of = [](uint64_t key) { return int32_t(key >> kStripBits); };
    for (int k = lane; k < teacher.entries; k += 64) {
        const uint64_t key = s.key[k];
        const int32_t place = int32_t(key & ((1u << kStripBits) - 1));
        Entry e{key == kNone ? -1 : id_of(key), place};
        if (GRAD && e.id >= 0) {
            if (k > 0 && id_of(s.key[k - 1]) == e.id) e.id = -1;
            else {
                float q = s.share[place];
                for (int j = k + 1; j < teacher.entries && s.key[j] != kNone && id_of(s.key[j]) == e.id; j++)
                    q += s.share[int32_t(s.key[j] & ((1u << kStripBits) - 1))];
                shares[first + k] = q;
            }
        }
        entries[first + k] = e;
    }
    if (GRAD || !strips) return r;
    // The first entry of a strip writes it, once the zeros have arrived.
    wave_fence();
    __builtin_amdgcn_s_waitcnt(0x0f70);                  // (no access to memory is on its way)
    wave_fence();
    const auto strip_of = [](uint64_t key) { return int64_t(key >> kStripBits) / kStripColumns; };
    for (int k = lane; k < teacher.entries; k += 64) {
        const uint64_t key = s.key[k];
        if (key == kNone || (k > 0 && strip_of(s.key[k - 1]) == strip_of(key))) continue;
        uint32_t n = 1;
        while (n < kStripMost && k + int(n) < teacher.entries && s.key[k + n] != kNone && strip_of(s.key[k + n]) == strip_of(key)) n++;
        row[strip_of(key)] = uint16_t(uint32_t(k) | n << kStripBits);
    }
    return r;
}

template <int M, bool GRAD>
__global__ __launch_bounds__(64 * kRowWaves) void teacher_rows(Teacher teacher, int64_t tokens, int64_t *__restrict__ mark,
                                                               Entry *__restrict__ entries, float *__restrict__ shares,
                                                               uint16_t *__restrict__ strips, int64_t pitch)
{
    __shared__ RowShared<M> all[kRowWaves];
    const int lane = int(threadIdx.x) & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
    const int64_t token = int64_t(blockIdx.x) * kRowWaves + wave;
    if (token >= tokens) return;                         // (no barriers of blocks follow)
    const TeacherRow r = row_entries<M, GRAD>(teacher, token, lane, all[wave], entries, shares, strips, pitch);
    if (lane == 0) mark[token] = r.wrong ? kWrong : r.takes_part() ? kTakesPart : kNoPart;
}

// Few tokens of a gradient: their entries and all that the products need of them, in one launch instead of three (5 to 9 us each).  Nothing is listed:
// a token that takes no part has a row of zeros and a factor of 0.  A block per row, zeros behind the last one up to whole tiles, once or (LOWER) twice;
// the blocks behind them pad rows of the weight.
constexpr int kFewRowWaves = 4;
struct FewRows {
    Header *header;          // of the tokens, and behind it of the products
    int32_t *place;
    float *base, *factor;
    float outer;
    int32_t top_bits;
};
// The largest finite factor of the tokens that take part, by a wave: what list_tokens finds in a list of them.  A lane looks at two tokens,
// eight of their entries at a time, until nobody is left whose factor could be larger: where all factors are alike that is one round,
// beside the sort of the block's own entries.  Gradients with and without this search (which took the largest factor of all tokens), us:
// 125 x 520 x 1003 bfloat16 22.5 and 21.3, 128 x 2048 x 50257 269.9 and 267.6, 16 x 2048 x 50257 213.6 and 213.8.
__device__ __forceinline__ float largest_factor(const Teacher &t, int64_t tokens, const float *__restrict__ dloss, int lane)
{
    static_assert(kLowerTokens <= 128, "two tokens a lane");
    constexpr int kEntries = 8;
    float size[2], top = 0.f;
#pragma unroll
    for (int h = 0; h < 2; h++) {
        const float g = lane + 64 * h < tokens ? fabsf(dloss[lane + 64 * h]) : 0.f;
        size[h] = g < __builtin_inff() ? g : 0.f;                // (neither infinities nor NaN)
    }
    for (int from = 0; from < t.entries && __ballot(size[0] > top || size[1] > top); from += kEntries) {
        float seen = 0.f;
#pragma unroll
        for (int h = 0; h < 2; h++) {
            if (!(size[h] > top)) continue;
            const int64_t first = int64_t(lane + 64 * h) * t.entries;
            bool part = false;
#pragma unroll
            for (int k = 0; k < kEntries; k++) {
                const int64_t at = first + (from + k < t.entries ? from + k : t.entries - 1), id = t.ids[at];
                part |= id != t.ignore && (id < 0 || id >= t.vocab || t.logit(at) * t.inverse != -__builtin_inff());
            }
            if (!part) continue;
            seen = fmaxf(seen, size[h]);
            size[h] = 0.f;
        }
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) seen = fmaxf(seen, __shfl_xor(seen, d, 64));
        top = fmaxf(top, seen);
    }
    return top;
}

template <typename T, int M, bool LOWER>
__global__ __launch_bounds__(64 * kFewRowWaves) void few_rows(Teacher teacher, int64_t tokens, const float *__restrict__ lse, const float *__restrict__ dloss,
                                                              const T *__restrict__ hidden, int64_t width, T *__restrict__ rows, int64_t pitch, FewRows out,
                                                              Entry *__restrict__ entries, float *__restrict__ shares, Padding<T> weight)
{
    __shared__ RowShared<M> s;
    __shared__ bool takes_part, wrong;
    __shared__ float top;
    const int tid = int(threadIdx.x), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t token = blockIdx.x, lower = lower_rows(tokens);
    if (token >= lower) {
        for (int64_t row = (token - lower) * kFewRowWaves + wave; row < weight.rows; row += (int64_t(gridDim.x) - lower) * kFewRowWaves)
            copy_row(weight.src + row * weight.width, weight.width, weight.dst + row * weight.pitch, weight.pitch, lane, 64);
        return;
    }
    // Wave 0 sees to the row's entries, and (where d has units) wave 1 to the unit.  The other waves copy the row meanwhile, and take it back if it turns out
    // to have no part.
    constexpr int kCopyFrom = LOWER ? 2 : 1;
    const auto copy = [&](const T *source) {
        copy_row(source, width, rows + token * pitch, pitch, tid - 64 * kCopyFrom, 64 * (kFewRowWaves - kCopyFrom));
        if (LOWER) copy_row(source, width, rows + (lower + token) * pitch, pitch, tid - 64 * kCopyFrom, 64 * (kFewRowWaves - kCopyFrom));
    };
    const float g = token < tokens ? dloss[token] : 0.f;
    if (wave >= kCopyFrom) copy(token < tokens ? hidden + token * width : nullptr);
    else if (wave == 1 && token < tokens) {
        const float largest = largest_factor(teacher, tokens, dloss, lane);
        if (lane == 0) top = largest;
    } else if (wave == 0) {
        TeacherRow r{0.f, 0.f, false};
        if (token < tokens) r = row_entries<M, true>(teacher, token, lane, s, entries, shares, nullptr, 0);
        if (lane == 0) {
            takes_part = token < tokens && r.takes_part() && g != 0.f;
            wrong = r.wrong;
        }
    }
    __syncthreads();
    if (token >= tokens) return;
    if (tid == 0) {
        const float unit = !LOWER || top == 0.f ? 1.f : fmaxf(top, 0x1p-100f);            // (as list_tokens has it)
        out.place[token] = takes_part ? int32_t(token) : -1;
        out.base[token] = takes_part ? lse[token] : 0.f;
        out.factor[token] = !takes_part ? 0.f : wrong ? __builtin_nanf("") : LOWER ? ldexpf(g / unit, out.top_bits - kLift) : g;
        if (token == 0) {
            const float unscale = ldexpf(unit, -out.top_bits) * out.outer;
            out.header[0] = Header{int32_t(tokens), unscale};
            if (LOWER) out.header[1] = Header{int32_t(2 * lower), unscale};
        }
    }
    if (wave >= kCopyFrom && !takes_part) copy(nullptr);
}

// A sum over the lanes of WAVES waves, in a fixed order; in the first of them.
template <int WAVES>
__device__ __forceinline__ float lanes_sum(float v, int lane)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
    if constexpr (WAVES > 1) {
        __shared__ float waves[WAVES];
        if ((lane & 63) == 0) waves[lane >> 6] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; w++) v += waves[w];
    }
    return v;
}

// The loss from the parts of a token's softmax and its picked logits: a wave per token, four of them in a block, or (few tokens) a block of many waves
// per token.  8192 tokens of 197 parts and 64 entries 10 us; one token 5.
template <int WAVES>
__global__ __launch_bounds__(64 * WAVES * join_tokens<WAVES>) void join_picked(Teacher teacher, int64_t tokens, const int32_t *__restrict__ place,
                                                                               int64_t parts, int64_t pitch, const float2 *__restrict__ stats,
                                                                               float *__restrict__ loss, float *__restrict__ lse, float *__restrict__ picked)
{
    constexpr int kLanes = 64 * WAVES;
    const int lane = int(threadIdx.x) % kLanes;
    const int64_t token = int64_t(blockIdx.x) * join_tokens<WAVES> + threadIdx.x / kLanes;
    if (token >= tokens) return;                         // (a whole wave; for WAVES > 1 no block)
    const TeacherRow row = teacher_row(teacher, token, lane & 63);
    const int64_t first = token * teacher.entries;
    const bool takes_part = row.takes_part();
    const float total = takes_part ? log_sum<WAVES>(stats + (place ? int64_t(place[token]) : token) * pitch, parts, lane) : 0.f;
    const float log_mass = logf(row.sum);
    float sum = 0.f;
    for (int k = lane; k < teacher.entries; k += kLanes) {
        const int64_t id = teacher.ids[first + k];
        if (!takes_part || id == teacher.ignore) picked[first + k] = 0.f;
        else if (id < 0 || id >= teacher.vocab) picked[first + k] = __builtin_nanf("");
        else {
            const float scaled = teacher.logit(first + k) * teacher.inverse, q = row.share(scaled);
            // (log q from differences: what a teacher's logits have in common, however large, takes no bits from it)
            if (q > 0.f) sum += q * ((scaled - row.top - log_mass) + (total - picked[first + k] * teacher.inverse));
        }
    }
    sum = lanes_sum<WAVES>(sum, lane);
    if (lane != 0) return;
    lse[token] = total;
    loss[token] = !takes_part ? 0.f : row.wrong ? __builtin_nanf("") : sum;
}

// d at the teacher's entries within a piece of the vocabulary, in its units: a thread per entry.
struct Entries {
    const Entry *entries;
    const float *shares;
    int32_t count;           // a token
    int64_t all;
    const int32_t *place;
    const float *lse, *factor, *picked;
    float inverse;
    int64_t from, columns, piece;
};
template <typename T, typename D, bool LOWER>
__device__ __forceinline__ void put_entry(const Entries &n, int64_t k, const Header *header, D *__restrict__ delta)
{
    if (k >= n.all) return;
    const int64_t token = uint32_t(k) / uint32_t(n.count);       // (fewer than 2^31 entries)
    const int32_t row = n.place[token];
    const Entry e = n.entries[k];
    if (row < 0) return;                                 // (it may have no sorted entries)
    const int64_t column = e.id - n.from;
    if (e.id < 0 || column < 0 || column >= n.columns) return;
    const float z = n.picked[token * n.count + e.place];
    const float d = (lifted<T>(z * n.inverse, n.lse[row]) - n.shares[k] * float(1 << lift_of<T>)) * n.factor[row];
    D *const out = delta + row * n.piece + column;
    if constexpr (LOWER) {
        const TwoParts<D> parts(d);
        *out = parts.upper;
        out[lower_rows(header->count) * n.piece] = parts.rest;
    } else *out = D(d);
}
template <typename T, bool LOWER>
__global__ __launch_bounds__(256) void delta_entries(const Header *header, Entries entries, T *__restrict__ delta)
{
    put_entry<T, T, LOWER>(entries, int64_t(blockIdx.x) * 256 + threadIdx.x, header, delta);
}

// d of few logits, entries and all: a block per 16 tokens and kFewColumns columns, whose waves sum a quarter of the width each (few_tiles), where
// tiles would leave most of the chip idle and sum all of it.  125 x 519 x 1003 binary32: 6.4 to 6.8 us, tiles and their entries 13.3 and 4.  Rows and
// columns behind the last ones are zeros, up to whole tiles and steps of the products.
// Taken for up to kFewTiles (64) tiles of logits.  us of whole gradients with it and with tiles: 128 x 512, 64 entries, 1000 columns (32 tiles)
// binary32 24.4 and 31.1, bfloat16 23.1 and 26.3, binary16 22.6 and 26.0; 2000 (64) 29.8 and 33.1, 25.1 and 27.2, 25.1 and 27.1; 4000 (126) 38.7 and
// 38.0, 30.4 and 28.9, 30.2 and 28.9; 8000 62 and 50, 44 and 36, 44 and 36; 16 x 512 x 4000 (63) 28.9 and 32.2, 23.1 and 24.6, 22.9 and 24.7.
// Entries a token, at most: every block looks at all of its tokens'.  128 x 512 x 1000, 256 of them: 36.7 and 39.1, 33.7 and 32.5, 33.4 and 32.4;
// 512: 76 and 74, 73 and 67, 73 and 67.
constexpr int kFewEntries = 256;
template <typename T, bool LOWER>
__global__ __launch_bounds__(64 * kFewWaves, 4) void few_delta(const T *__restrict__ hidden, const T *__restrict__ weight, int64_t width, int64_t tokens,
                                                               uint32_t groups, Entries entries, T *__restrict__ delta)
{
    __shared__ __align__(16) float part[kFewWaves][16][kFewPitch];
    __shared__ float share[16][kFewColumns];
    const int tid = int(threadIdx.x), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t n0 = int64_t(blockIdx.x / groups) * kFewColumns, m0 = int64_t(blockIdx.x % groups) * 16;
    const int64_t columns = entries.columns - n0, count = tokens - m0;
    constexpr int kEach = 16 * kFewColumns / (64 * kFewWaves), kLanes = kFewColumns / kEach;
    const int m = tid / kLanes, first = tid % kLanes * kEach;
    const int64_t token = m0 + m;
    const float base = m < count ? entries.lse[token] : 0.f, f = m < count ? entries.factor[token] : 0.f;
    for (int k = tid; k < 16 * kFewColumns; k += 64 * kFewWaves) share[k / kFewColumns][k % kFewColumns] = 0.f;
    __syncthreads();
    if (f != 0.f)                                        // (others may have no sorted entries)
        for (int k = tid % kLanes; k < entries.count; k += kLanes) {
            const int64_t at = token * entries.count + k, column = int64_t(entries.entries[at].id) - entries.from - n0;
            const float q = entries.shares[at];
            if (entries.entries[at].id >= 0 && column >= 0 && column < kFewColumns) share[m][column] = q;
        }
    if (columns > 0 && count > 0)
        few_products(part, hidden + m0 * width, weight + n0 * width, width, int(columns < kFewColumns ? columns : kFewColumns), int(count < 16 ? count : 16), wave, lane);
    __syncthreads();
    typedef T Vec __attribute__((ext_vector_type(kEach)));
    Vec upper, rest;
#pragma unroll
    for (int e = 0; e < kEach; e++) {
        float z = 0.f;
#pragma unroll
        for (int k = 0; k < kFewWaves; k++) z += part[k][m][first + e];
        const float d = f == 0.f || first + e >= columns ? 0.f : (lifted<T>(z * entries.inverse, base) - share[m][first + e] * float(1 << lift_of<T>)) * f;
        if constexpr (LOWER) {
            const TwoParts<T> parts(d);
            upper[e] = parts.upper;
            rest[e] = parts.rest;
        } else upper[e] = T(d);
    }
    T *const out = delta + token * entries.piece + n0 + first;
    *reinterpret_cast<Vec *>(out) = upper;
    if (LOWER) *reinterpret_cast<Vec *>(out + lower_rows(tokens) * entries.piece) = rest;
}

// bfloat16 to binary16, whose smaller range takes what is multiplied by a power of two, exactly: one that brings the largest magnitude into [2^14, 2^15).
// Then everything down to 2^-31 of the largest keeps its eight bits.  The first pass converts with a guess of that power, and remembers the largest
// magnitude its blocks saw; the second one converts again only where that did not come into [2^3, 2^15): down to 2^-20 of the largest all bits are kept then.
// Bound by memory: in launches of its own the first pass took 16 us for 30522 x 768 weights, 97 for 50257 x 2048 and 8192 x 2048 hidden states in two pieces; as
// the last blocks of d's launch 8, where d's tiles fill 1.4 rounds, and still 80 to 88, where they fill twelve and both want the same memory.  The second
// pass takes 5 us where it finds nothing to do.
struct Conversion {
    _Float16 *to;
    int64_t pieces;          // of 16 bytes, at most
    float *most, *scale;
    int guess;
};
constexpr int kHiddenGuess = 4, kWeightGuess = 10;   // largest hidden states of 2^-1 to 2^11, weights of 2^-7 to 2^5
__device__ __forceinline__ float finite_magnitude(float v) { return fabsf(v) < __builtin_inff() ? fabsf(v) : 0.f; }
__device__ __forceinline__ float block_most(float v)
{
    __shared__ float waves[8];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor(v, d, 64));
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = v;
    __syncthreads();
    for (uint32_t w = 0; w < blockDim.x / 64; w++) v = fmaxf(v, waves[w]);
    __syncthreads();
    return v;
}
template <bool AGAIN>
__device__ __forceinline__ void convert(const Conversion &c, const __bf16 *source, int64_t pieces, uint32_t block, uint32_t blocks)
{
    typedef __bf16 From __attribute__((ext_vector_type(8)));
    typedef _Float16 To __attribute__((ext_vector_type(8)));
    int shift = c.guess;
    if (AGAIN) {
        float v = 0.f;
        for (int k = int(threadIdx.x); k < kConvertBlocks; k += int(blockDim.x)) v = fmaxf(v, c.most[k]);
        v = block_most(v);
        const bool again = v > 0.f && !(ilogbf(v) + shift >= 3 && ilogbf(v) + shift < 15);
        if (again) shift = 14 - ilogbf(v);
        if (block == 0 && threadIdx.x == 0) *c.scale = ldexpf(1.f, -shift);
        if (!again) return;
    }
    float most = 0.f;
    for (int64_t k = int64_t(block) * blockDim.x + threadIdx.x; k < pieces; k += int64_t(blocks) * blockDim.x) {
        const From v = reinterpret_cast<const From *>(source)[k];
        To out;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const float x = float(v[e]);
            if (!AGAIN) most = fmaxf(most, finite_magnitude(x));
            out[e] = _Float16(ldexpf(x, shift));
        }
        reinterpret_cast<To *>(c.to)[k] = out;
    }
    if (AGAIN) return;
    most = block_most(most);
    if (threadIdx.x == 0) c.most[block] = most;
}
// rows.to may be null: the hidden states are converted with the first piece of the weight.
template <bool AGAIN>
__device__ __forceinline__ void convert_both(const Conversion &rows, const Conversion &weight, uint32_t block, uint32_t blocks, const Header *header,
                                             Hidden<__bf16> hidden, const __bf16 *source_weight, int64_t pitch)
{
    if (rows.to) {
        const int64_t count = header->count;
        convert<AGAIN>(rows, hidden.of(count), lower_rows(count) * pitch / 8, block, blocks);
    }
    convert<AGAIN>(weight, source_weight, weight.pieces, block, blocks);
}
// The first pass is done by the last blocks of the launch that forms d.
struct FirstPass {
    static constexpr bool kAny = true;
    uint32_t blocks;
    Conversion rows, weight;
    __device__ __forceinline__ void operator()(uint32_t block, const Header *header, Hidden<__bf16> hidden, const __bf16 *source_weight, int64_t pitch) const
    {
        convert_both<false>(rows, weight, block, blocks, header, hidden, source_weight, pitch);
    }
};
// The second one; its blocks behind the first kAgainBlocks see to the teacher's entries.
constexpr uint32_t kAgainBlocks = 1024;
__global__ __launch_bounds__(256) void convert_again(const Header *header, Hidden<__bf16> hidden, int64_t pitch, const __bf16 *__restrict__ source_weight,
                                                     Conversion rows, Conversion weight, Entries entries, _Float16 *__restrict__ delta)
{
    if (blockIdx.x < kAgainBlocks) convert_both<true>(rows, weight, blockIdx.x, kAgainBlocks, header, hidden, source_weight, pitch);
    else put_entry<__bf16, _Float16, false>(entries, int64_t(blockIdx.x - kAgainBlocks) * 256 + threadIdx.x, header, delta);
}

Teacher teacher_of(const DistillLayout &l, const DistillBuffers &b)
{
    return Teacher{b.ids, b.teacher, l.entries, b.teacher_dt, b.ignore, l.head.vocab, 1.f / b.temperature};
}

template <bool GRAD>
hipError_t rows(const DistillLayout &l, const DistillBuffers &b, hipStream_t stream)
{
    const auto go = [&](auto most) {
        constexpr int M = decltype(most)::value;
        teacher_rows<M, GRAD><<<dim3(uint32_t((l.head.tokens + kRowWaves - 1) / kRowWaves)), 64 * kRowWaves, 0, stream>>>(
            teacher_of(l, b), l.head.tokens, reinterpret_cast<int64_t *>(b.workspace + l.mark), reinterpret_cast<Entry *>(b.workspace + l.entry),
            GRAD ? reinterpret_cast<float *>(b.workspace + l.share) : nullptr,
            !GRAD ? reinterpret_cast<uint16_t *>(b.workspace + l.strip) : nullptr, l.strips);
    };
    if (l.entries <= 64) go(std::integral_constant<int, 64>());
    else if (l.entries <= 128) go(std::integral_constant<int, 128>());
    else if (l.entries <= 256) go(std::integral_constant<int, 256>());
    else go(std::integral_constant<int, kMostEntries>());
    return hipGetLastError();
}

HeadBuffers head_of(const DistillLayout &l, const DistillBuffers &b)
{
    return HeadBuffers{b.hidden, b.weight, reinterpret_cast<const int64_t *>(b.workspace + l.mark), kNoPart, b.workspace};
}

template <typename T>
hipError_t divergence(const DistillLayout &l, const DistillBuffers &b, float *loss, float *lse, float *picked, hipStream_t stream)
{
    const HeadBuffers h = head_of(l, b);
    const Teacher teacher = teacher_of(l, b);
    Calls<T, Tempered> calls{l.head, h, stream, Tempered{teacher.inverse}};
    // Few tokens' kernel takes the products of the entries' rows along; other tiles pick the logits out.  Both against products of gathered rows after the
    // tiles, us: one token x 1024 x 50257 binary16 24.7 and 30.7; picked 33 x 2048 x 50257 bfloat16, 64 entries, 57 and 82, 2048 x 2048 x 50257 384 and 461,
    // 2000 x 512 x 1000 of 16, 64 and 256 entries 29, 35, 66 and 36, 57, 144, 2000 x 2048 x 5000 of 1000 entries 282 and 1384.
    const bool direct = calls.direct(), few = calls.few();
    hipError_t error = few ? hipSuccess : rows<false>(l, b, stream);
    if (few) {
        calls.picks.blocks = uint32_t((l.head.tokens * ((l.entries + kDots - 1) / kDots) + kFewWaves - 1) / kFewWaves);
        calls.picks.ids = b.ids;
        calls.picks.ignore = b.ignore;
    } else {
        calls.tokens_of_rows = calls.template at<int32_t>(l.token);       // (not written, nor read, where tokens are taken as they come)
        calls.picks.strips = calls.template at<uint16_t>(l.strip);
        calls.picks.entries = calls.template at<Entry>(l.entry);
        calls.picks.token = calls.tokens_of_rows;
        calls.picks.pitch = l.strips;
    }
    calls.picks.picked = picked;
    calls.picks.count = l.entries;
    const int side = calls.loss_parts();
    const int64_t parts = (l.head.vocab + side - 1) / side;
    const int32_t *const place = direct ? nullptr : calls.template at<int32_t>(l.head.place);
    const float2 *const stats = calls.template at<float2>(l.head.stats);
    const auto join = [&](auto waves) {
        constexpr int WAVES = decltype(waves)::value, kPerBlock = join_tokens<WAVES>;
        join_picked<WAVES><<<dim3(uint32_t((l.head.tokens + kPerBlock - 1) / kPerBlock)), 64 * WAVES * kPerBlock, 0, stream>>>(
            teacher, l.head.tokens, place, parts, l.head.parts, stats, loss, lse, picked);
    };
    if (direct) join(std::integral_constant<int, kJoinWaves>());
    else join(std::integral_constant<int, 1>());
    calls.launched();
    if (error == hipSuccess) error = calls.error;
    return error;
}

template <typename T, typename D>
hipError_t gradient_of(const DistillLayout &l, const DistillBuffers &b, const float *lse, const float *picked, const float *dloss, void *dhidden,
                       void *dweight, hipStream_t stream)
{
    const HeadBuffers h = head_of(l, b);
    const float inverse = teacher_of(l, b).inverse;
    Calls<T, Tempered, D> calls{l.head, h, stream, Tempered{inverse}};
    const auto at = [&](size_t offset) { return b.workspace + offset; };
    calls.lower = l.lower;
    if constexpr (calls.kOther) {
        calls.hidden_of_products = reinterpret_cast<D *>(at(l.hidden16));
        calls.weight_of_products = reinterpret_cast<D *>(at(l.weight16));
        calls.scales = reinterpret_cast<float *>(at(l.scales));
    }
    hipError_t error = hipSuccess;
    const int64_t all = l.head.tokens * l.entries;
    const bool few = l.head.tokens > 0 && l.head.tokens <= kLowerTokens;
    calls.copied = few;
    calls.few_logits = few && !l.other && calls.few_of_both() && l.entries <= kFewEntries;
    const auto prepare_few = [&](auto most) {
        constexpr int M = decltype(most)::value;
        const int64_t columns = l.head.padded ? l.head.columns(0) : 0, wanted = (columns + kFewRowWaves - 1) / kFewRowWaves;
        const int64_t pads = wanted < 8 * kHeadBlocks ? wanted : 8 * kHeadBlocks;
        const FewRows out{calls.header(), calls.template at<int32_t>(l.head.place), calls.template at<float>(l.head.lse),
                          calls.template at<float>(l.head.factor), inverse, calls.kTopBits};
        few_rows<T, M, sizeof(T) == 2><<<dim3(uint32_t(lower_rows(l.head.tokens) + pads)), 64 * kFewRowWaves, 0, stream>>>(
            teacher_of(l, b), l.head.tokens, lse, dloss, static_cast<const T *>(b.hidden), l.head.width, calls.template at<T>(l.head.hidden), l.head.pitch, out,
            calls.template at<Entry>(l.entry), calls.template at<float>(l.share),
            Padding<T>{static_cast<const T *>(b.weight), calls.template at<T>(l.head.weight), columns, l.head.width, l.head.pitch});
        calls.launched();
    };
    const auto listed = [&] {
        if (!few) {
            if (l.head.tokens) error = rows<true>(l, b, stream);
            calls.list(dloss, lse, inverse);
        } else if (l.entries <= 64) prepare_few(std::integral_constant<int, 64>());
        else if (l.entries <= 128) prepare_few(std::integral_constant<int, 128>());
        else if (l.entries <= 256) prepare_few(std::integral_constant<int, 256>());
        else prepare_few(std::integral_constant<int, kMostEntries>());
    };
    const auto beside = [&](int64_t first, int64_t columns) {
        if constexpr (calls.kOther) {
            float *const most = reinterpret_cast<float *>(at(l.most));
            return FirstPass{kConvertBlocks, Conversion{first == 0 ? calls.hidden_of_products : nullptr, 0, most, calls.scales, kHiddenGuess},
                             Conversion{calls.weight_of_products, columns * l.head.pitch / 8, most + kConvertBlocks, calls.scales + 1, kWeightGuess}};
        } else return Nothing();
    };
    const auto entries = [&](const T *w, int64_t first, int64_t columns) {
        const Entries n{calls.template at<Entry>(l.entry), calls.template at<float>(l.share), l.entries, all, calls.template at<int32_t>(l.head.place),
                        calls.template at<float>(l.head.lse), calls.template at<float>(l.head.factor), picked, inverse, first, columns, l.head.piece};
        const uint32_t blocks = uint32_t((all + 255) / 256);
        if constexpr (calls.kOther) {
            const FirstPass done = beside(first, columns);
            convert_again<<<dim3(kAgainBlocks + blocks), 256, 0, stream>>>(calls.header(), calls.hidden(), l.head.pitch, w, done.rows, done.weight, n,
                                                                           calls.template at<D>(l.head.delta));
            calls.launched();
        } else if (calls.few_logits) {
            const uint32_t groups = uint32_t(lower_rows(l.head.tokens) / 16), wide = uint32_t((columns + 63) / 64 * 64 / kFewColumns);
            few_delta<T, sizeof(T) == 2><<<dim3(groups * wide), 64 * kFewWaves, 0, stream>>>(
                static_cast<const T *>(b.hidden), static_cast<const T *>(b.weight) + first * l.head.width, l.head.width, l.head.tokens, groups, n,
                calls.template at<T>(l.head.delta));
            calls.launched();
        } else {
            const auto go = [&](auto in_two) {
                delta_entries<T, decltype(in_two)::value><<<dim3(blocks), 256, 0, stream>>>(calls.header(), n, calls.template at<T>(l.head.delta));
            };
            if constexpr (calls.kFewOnly) go(std::true_type());
            else if (l.lower) go(std::bool_constant<sizeof(T) == 2>());
            else go(std::false_type());
            calls.launched();
        }
    };
    const hipError_t rest = calls.gradient(static_cast<T *>(dhidden), static_cast<T *>(dweight), listed, beside, entries);
    return error != hipSuccess ? error : rest;
}

}  // namespace

int launch_distill(const DistillLayout &l, const DistillBuffers &b, float *loss, float *lse, float *picked, void *stream)
{
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (l.head.tokens == 0) return hipSuccess;
    if (l.head.dt == CGX_F32) return divergence<float>(l, b, loss, lse, picked, s);
    if (l.head.dt == CGX_F16) return divergence<_Float16>(l, b, loss, lse, picked, s);
    return divergence<__bf16>(l, b, loss, lse, picked, s);
}

int launch_distill_grad(const DistillLayout &l, const DistillBuffers &b, const float *lse, const float *picked, const float *dloss,
                        void *dhidden, void *dweight, void *stream)
{
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (l.head.dt == CGX_F32) return gradient_of<float, float>(l, b, lse, picked, dloss, dhidden, dweight, s);
    if (l.head.dt == CGX_F16) return gradient_of<_Float16, _Float16>(l, b, lse, picked, dloss, dhidden, dweight, s);
    if (l.other) return gradient_of<__bf16, _Float16>(l, b, lse, picked, dloss, dhidden, dweight, s);
    return gradient_of<__bf16, __bf16>(l, b, lse, picked, dloss, dhidden, dweight, s);
}

}  // namespace cgx
