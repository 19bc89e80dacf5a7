// The embedding's kernels and their launches: rows of a table for a list of tokens, and the table's gradient.
//
//   lookup    out[n] = scale table[ids[n]]
//   gradient  dtable[v] = scale sum_{n: ids[n] = v} dout[n]  (+ dtable[v])
// Both are bound by memory: an element read or written costs less than one vector instruction.  The gradient's sums are taken in the order of
// the tokens sorted by id, so that a row is written once, by one wave, and no atomics are needed: the same call gives the same bits.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "cgx_embed.h"

namespace cgx {
namespace {

constexpr int kBlock = 256;

struct EmbedHeader {
    int32_t count;           // tokens that take part
};

// 16 bytes of a row, V elements; rows start at any element.
template <typename T>
struct Piece {
    static constexpr int V = 16 / int(sizeof(T));
    typedef T Vec __attribute__((ext_vector_type(V)));
    typedef Vec Anywhere __attribute__((aligned(sizeof(T))));
    static __device__ __forceinline__ Vec load(const T *row, int64_t column, int64_t width)
    {
        if (column + V <= width) return *reinterpret_cast<const Anywhere *>(row + column);
        Vec v = Vec(T(0.f));
#pragma unroll
        for (int e = 0; e < V; e++)
            if (column + e < width) v[e] = row[column + e];
        return v;
    }
    static __device__ __forceinline__ void store(T *row, int64_t column, int64_t width, Vec v)
    {
        if (column + V <= width) {
            *reinterpret_cast<Anywhere *>(row + column) = v;
            return;
        }
#pragma unroll
        for (int e = 0; e < V; e++)
            if (column + e < width) row[column + e] = v[e];
    }
};

// ---------------------------------------------------------------- lookup

// A wave takes EACH strips (of 64 x 16 bytes) of a row, all of them on their way at a time: as many as leave a wave for every place on the chip, since
// an id, its row and the store are three dependent steps.  8192 x 2048 of 50257 bfloat16 10.8 us (67 MB read and written, 6.2 TB/s); one token 1.6 us.
template <typename T, int EACH>
__global__ __launch_bounds__(kBlock) void look_up(const T *__restrict__ table, const int64_t *__restrict__ ids, int64_t tokens, int64_t width,
                                                  int64_t vocab, int64_t ignore, float scale, uint32_t parts, T *__restrict__ out)
{
    using P = Piece<T>;
    const int lane = int(threadIdx.x) & 63;
    const int64_t item = int64_t(blockIdx.x) * (kBlock / 64) + __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
    const int64_t token = item / parts, first = (item % parts * EACH * 64 + lane) * P::V;
    if (token >= tokens) return;
    const int64_t id = ids[token];
    const bool there = id >= 0 && id < vocab && id != ignore;
    const float otherwise = id == ignore ? 0.f : __builtin_nanf("");
    const T *row = table + (there ? id : 0) * width;
    T *const to = out + token * width;
    typename P::Vec v[EACH];
#pragma unroll
    for (int k = 0; k < EACH; k++) {
        const int64_t column = first + k * 64 * P::V;
        if (there && column < width) v[k] = P::load(row, column, width);
    }
#pragma unroll
    for (int k = 0; k < EACH; k++) {
        const int64_t column = first + k * 64 * P::V;
        if (column >= width) break;
        typename P::Vec r;
#pragma unroll
        for (int e = 0; e < P::V; e++) r[e] = T(there ? float(v[k][e]) * scale : otherwise);
        P::store(to, column, width, r);
    }
}

// ---------------------------------------------------------------- gradient: tokens sorted by id

constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64, kSortEach = 8, kDigitBits = 8, kDigits = 1 << kDigitBits, kVotedBits = 3;

struct SortShared {
    uint32_t place[kSortWaves][kDigits];     // entries of a digit in a wave's part, then where the next one of them goes
    uint32_t waves[kDigits / 64], ahead[kSortWaves], all;
};

__device__ __forceinline__ uint32_t wave_sum(uint32_t v)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
    return v;
}

// A wave's walk over entries `from` to `to` of a list, 64 at a time: `visit(entry, i, exists)`, called by all lanes.  All loads first, of entries that
// exist: none waits for another one's condition.
template <class Load, class Visit>
__device__ __forceinline__ void walk(uint32_t from, uint32_t to, int lane, Load load, Visit visit)
{
    for (uint32_t i = from; i < to; i += 64 * kSortEach) {
        decltype(load(0u)) entry[kSortEach];
#pragma unroll
        for (int k = 0; k < kSortEach; k++) {
            const uint32_t at = i + 64 * k + lane;
            entry[k] = load(at < to ? at : to - 1);
        }
#pragma unroll
        for (int k = 0; k < kSortEach; k++) visit(entry[k], i + 64 * k + lane, i + 64 * k + lane < to);
    }
}
// The walk of a wave's share of n entries: a run of neighbouring ones.
// (Keeping up to 8192 entries in registers from the first walk to the second one took 3 us more for 8192 tokens, and as much for 4096.)
template <class Load>
struct Run {
    uint32_t from, to;
    Load load;
    __device__ __forceinline__ Run(uint32_t n, int wave, Load l) : load(l)
    {
        const uint32_t each = ((n + kSortWaves - 1) / kSortWaves + 63) / 64 * 64;
        from = uint32_t(wave) * each;
        to = from + each < n ? from + each : n;
    }
    template <class Visit>
    __device__ __forceinline__ void operator()(int lane, Visit visit) const { walk(from, to, lane, load, visit); }
};

// One stable pass of a sort by digits, by a block.  `run(lane, visit)` walks over a wave's entries, those of the waves one after another; `read(entry, i,
// exists, key, token)` says whether an entry takes part, and `write(place, key, token)` gets the entries in the order of the digit `key >> shift`, those of
// one digit in the order they come in.  `counted(n)` is called by all threads between the two walks; thread 0's argument is how many take part.  Ranks
// within a digit follow from the counts of the waves before and, among a wave's own 64 at a time, from votes.
template <class Walk, class Read, class Counted, class Write>
__device__ __forceinline__ void sort_pass(SortShared &s, int shift, int bits, Walk run, Read read, Counted counted, Write write)
{
    const int tid = int(threadIdx.x), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t mask = (1u << bits) - 1;
    for (int k = tid; k < kSortWaves * kDigits; k += kSortThreads) s.place[k / kDigits][k % kDigits] = 0;
    __syncthreads();
    const auto lanes_of = [&](uint32_t digit, uint64_t same) {
        for (int b = 0; b < bits; b++) {
            const uint64_t ones = __ballot((digit >> b) & 1);
            same &= (digit >> b) & 1 ? ones : ~ones;
        }
        return same;
    };
    const auto rank_of = [](uint64_t same) { return __builtin_amdgcn_mbcnt_hi(uint32_t(same >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(same), 0u)); };
    run(lane, [&](auto entry, uint32_t i, bool exists) {
        uint32_t key;
        int32_t token;
        const bool in = read(entry, i, exists, key, token);
        const uint32_t digit = (key >> shift) & mask;
        // (additions to one address are made one after another: few digits are counted by votes.  65536 tokens of 259 entries: 20 and 17 us)
        if (bits > kVotedBits) {
            if (in) atomicAdd(&s.place[wave][digit], 1u);
        } else {
            const uint64_t same = lanes_of(digit, __ballot(in));
            if (in && rank_of(same) == 0) atomicAdd(&s.place[wave][digit], uint32_t(__popcll(same)));
        }
    });
    __syncthreads();
    // places: digits in order, the waves of a digit in order
    uint32_t mine = 0, before = 0, sum = 0;
    if (tid < kDigits) {
        for (int w = 0; w < kSortWaves; w++) mine += s.place[w][tid];
        before = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t other = __shfl_up(before, d, 64);
            before += lane >= d ? other : 0;
        }
        if (lane == 63) s.waves[wave] = before;
    }
    __syncthreads();
    for (int w = 0; w < kDigits / 64; w++) sum += s.waves[w];
    if (tid < kDigits) {
        before -= mine;
        for (int w = 0; w < wave; w++) before += s.waves[w];
        for (int w = 0; w < kSortWaves; w++) {
            const uint32_t here = s.place[w][tid];
            s.place[w][tid] = before;
            before += here;
        }
    }
    counted(sum);
    __syncthreads();
    run(lane, [&](auto entry, uint32_t i, bool exists) {
        uint32_t key;
        int32_t token;
        const bool in = read(entry, i, exists, key, token);
        const uint64_t vote = __ballot(in);
        if (!vote) return;
        const uint32_t digit = (key >> shift) & mask;
        const uint64_t same = lanes_of(digit, vote);
        if (in) {
            const uint32_t rank = rank_of(same);
            const uint32_t first = s.place[wave][digit];
            write(first + rank, key, token);
            __builtin_amdgcn_wave_barrier();
            if (rank == 0) s.place[wave][digit] = first + uint32_t(__popcll(same));
            __builtin_amdgcn_wave_barrier();
        }
    });
    __syncthreads();
}

// Lists are read and written with offsets of 32 bits from a uniform address: they have fewer than 2^24 entries.
template <typename U>
__device__ __forceinline__ U &listed(U *list, uint32_t at)
{
    using Bytes = std::conditional_t<std::is_const<U>::value, const unsigned char, unsigned char>;
    return *reinterpret_cast<U *>(reinterpret_cast<Bytes *>(list) + at * uint32_t(sizeof(U)));
}

// Ids of a share [from, from + span) of the vocabulary.  Few instructions: every block does this for every token.
struct Id {
    uint32_t low, high;
};
struct Share {
    uint32_t from, span, mark;
    bool marked;             // `ignore` is an entry of the vocabulary
    __device__ __forceinline__ Share(int64_t low, int64_t high, int64_t vocab, int64_t ignore)
        : from(uint32_t(low)), span(uint32_t(high - low)), mark(uint32_t(ignore)), marked(ignore >= 0 && ignore < vocab) {}
    __device__ __forceinline__ bool valid(Id id) const { return id.high == 0 && !(marked && id.low == mark); }       // (or beyond the vocabulary)
    __device__ __forceinline__ uint32_t key(Id id) const { return id.low - from; }
    __device__ __forceinline__ bool has(Id id) const { return valid(id) && key(id) < span; }
};

// Many tokens: first, blocks sort a part of them each by share.  starts[share][part]: where a share begins in a part.
struct Parts {
    SortedToken *list;
    uint32_t *starts;
    uint32_t each;           // tokens of a part
    int32_t share_bits;
};
__global__ __launch_bounds__(kSortThreads) void sort_parts(const int64_t *__restrict__ ids, uint32_t tokens, int64_t ignore, int64_t vocab, int32_t shares, Parts parts)
{
    __shared__ SortShared s;
    const int tid = int(threadIdx.x), wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t first = blockIdx.x * parts.each < tokens ? blockIdx.x * parts.each : tokens, n = tokens - first < parts.each ? tokens - first : parts.each;
    const Share all(0, vocab, vocab, ignore);
    const Id *const own = reinterpret_cast<const Id *>(ids) + first;
    sort_pass(
        s, parts.share_bits, kDigitBits, Run(n, wave, [&](uint32_t i) { return listed(own, i); }),
        [&](Id id, uint32_t i, bool exists, uint32_t &key, int32_t &token) {
            key = id.low;
            token = int32_t(first + i);
            return exists && all.has(id);
        },
        [&](uint32_t count) {
            // (a digit's places have been written by this thread)
            if (tid < shares && tid < kDigits) parts.starts[tid * kEmbedParts + blockIdx.x] = s.place[0][tid];
            if (tid == 0) parts.starts[shares * kEmbedParts + blockIdx.x] = count;
        },
        [&](uint32_t place, uint32_t key, int32_t token) {
            if (place < n) listed(parts.list + first, place) = SortedToken{int32_t(key), token};
        });
}

// The first sort_blocks blocks sort the tokens of a share of the vocabulary each, stably, eight bits of their place in the share at a time (one pass for up
// to 65536 entries).  Up to some thousand tokens a block finds its own by looking at all ids, and learns from them how many there are ahead of it
// (PARTS false); these 256 looks at every token cost more than a launch from kEmbedManyTokens on, where it takes its share from every part instead.
// The blocks behind them write zeros over the table meanwhile, which hides the sort wherever the table is long.
// 65536 tokens of 259 entries: 36 us looking at all ids, whether 8 or 16 loads of a lane are on their way, and with half the instructions: 128 visits of 64
// ids by each of a block's waves; 23 us in parts, the longest share (a fifth of the tokens) in 17 of them.  Whole gradients of 256 columns looking at all
// ids and in parts: 16384 tokens 30.5 and 36.0 us, 32768 41.9 and 37.4, 65536 65 and 45, alike for 259, 5000 and 50257 entries.
// Zeros alone: 206 MB in 26 us into the memory-side cache, in some 40 past it.
// (Without a limit of its registers: 41 to 59 of them, no scratch memory.  A build that was forced to spill some faulted, its cause is not known.)
constexpr int kFillBytes = 64 << 10;                 // of the table, a block
template <bool FILL, bool PARTS>
__global__ __launch_bounds__(kSortThreads) void sort_tokens(const int64_t *__restrict__ ids, uint32_t tokens, int64_t ignore, int64_t vocab,
                                                            int64_t share, int32_t bits, uint32_t sort_blocks, EmbedHeader *header,
                                                            SortedToken *list, SortedToken *between, Parts parts,
                                                            unsigned char *__restrict__ table, int64_t bytes)
{
    const int tid = int(threadIdx.x), wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if (FILL && blockIdx.x >= sort_blocks) {
        typedef uint32_t Vec __attribute__((ext_vector_type(4)));
        const int64_t first = int64_t(blockIdx.x - sort_blocks) * kFillBytes;
#pragma unroll
        for (int k = 0; k < kFillBytes / (16 * kSortThreads); k++) {
            const int64_t at = first + (int64_t(k) * kSortThreads + tid) * 16;
            if (at + 16 <= bytes) *reinterpret_cast<Vec *>(table + at) = Vec(0u);
            else
                for (int64_t b = at; b < bytes; b += 2) *reinterpret_cast<uint16_t *>(table + b) = 0;       // (elements of 2 or 4 bytes)
        }
        return;
    }
    __shared__ SortShared s;
    const int64_t low = int64_t(blockIdx.x) * share, high = low + share < vocab ? low + share : vocab;
    const Share own(low, high, vocab, ignore);
    const int passes = bits <= kDigitBits ? 1 : (bits + kDigitBits - 1) / kDigitBits, first_bits = bits < kDigitBits ? bits : kDigitBits;
    uint32_t base = 0, mine = 0;
    SortedToken *to = passes % 2 ? list : between;
    const auto put = [&](uint32_t place, uint32_t key, int32_t token) {
        const uint32_t at = base + place;
        if (at < tokens) listed(to, at) = SortedToken{int32_t(own.from + key), token};       // (even if ids change between two walks over them)
    };
    const auto from_list = [&](SortedToken e, uint32_t, bool exists, uint32_t &key, int32_t &token) {
        key = uint32_t(e.id) - own.from;
        token = e.token;
        return exists;
    };
    // What is ahead of the share, a sum over the block, and how many tokens it has (thread 0 says), in every thread.
    const auto totals = [&](uint32_t ahead, uint32_t count) {
        const uint32_t x = wave_sum(ahead);
        if ((tid & 63) == 0) s.ahead[tid >> 6] = x;
        if (tid == 0) s.all = count;
        __syncthreads();
        for (int w = 0; w < kSortWaves; w++) base += s.ahead[w];
        mine = s.all;
        if (blockIdx.x == sort_blocks - 1 && tid == 0) header->count = int32_t(base + mine);
    };
    if constexpr (PARTS) {
        __shared__ uint32_t start[kEmbedParts], length[kEmbedParts];
        uint32_t from = 0, n = 0;
        if (tid < kEmbedParts) {
            from = parts.starts[blockIdx.x * kEmbedParts + tid];
            n = parts.starts[(blockIdx.x + 1) * kEmbedParts + tid] - from;
            start[tid] = uint32_t(tid) * parts.each + from;
            length[tid] = n;
        }
        const uint32_t count = wave_sum(n);
        if ((tid & 63) == 0 && tid < kEmbedParts) s.waves[tid >> 6] = count;
        __syncthreads();
        uint32_t all = 0;
        for (int w = 0; w < kEmbedParts / 64; w++) all += s.waves[w];
        totals(from, all);                               // (what is ahead of this share in every part)
        // Neighbouring parts a wave: what several of them begin with, up to 64 each, is on its way at a time.
        const auto load = [&](uint32_t at) { return listed(parts.list, at < tokens ? at : 0u); };
        const auto run = [&](int lane, auto visit) {
            constexpr int kEach = kEmbedParts / kSortWaves;
            for (int p0 = wave * kEach; p0 < (wave + 1) * kEach; p0 += kSortEach) {
                SortedToken entry[kSortEach];
#pragma unroll
                for (int k = 0; k < kSortEach; k++) entry[k] = load(start[p0 + k] + (uint32_t(lane) < length[p0 + k] ? lane : 0));
#pragma unroll
                for (int k = 0; k < kSortEach; k++) {
                    const uint32_t first = start[p0 + k], here = __builtin_amdgcn_readfirstlane(length[p0 + k]);
                    visit(entry[k], 0u, uint32_t(lane) < here);
                    if (here > 64) walk(64, here, lane, [&](uint32_t i) { return load(first + i); }, visit);
                }
            }
        };
        sort_pass(s, 0, first_bits, run, from_list, [](uint32_t) {}, put);
    } else {
        uint32_t ahead = 0;
        bool counting = true;
        const Id *const all = reinterpret_cast<const Id *>(ids);
        const auto from_ids = [&](Id id, uint32_t i, bool exists, uint32_t &key, int32_t &token) {
            const bool valid = exists && own.valid(id);
            if (counting) ahead += valid && id.low < own.from;
            key = own.key(id);
            token = int32_t(i);
            return valid && key < own.span;
        };
        sort_pass(
            s, 0, first_bits, Run(tokens, wave, [&](uint32_t i) { return listed(all, i); }), from_ids,
            [&](uint32_t count) {
                counting = false;
                totals(ahead, count);
            },
            put);
    }
    for (int p = 1; p < passes; p++) {
        SortedToken *const from = to + base;
        to = to == list ? between : list;
        const int left = bits - p * kDigitBits;
        sort_pass(s, p * kDigitBits, left < kDigitBits ? left : kDigitBits, Run(mine, wave, [&](uint32_t i) { return listed(from, i); }), from_list,
                  [](uint32_t) {}, put);
    }
}

// ---------------------------------------------------------------- gradient: sums

template <typename T>
__device__ __forceinline__ void finish(const float (&acc)[Piece<T>::V], float scale, bool accumulate, T *row, int64_t column, int64_t width)
{
    using P = Piece<T>;
    typename P::Vec v;
    if (accumulate) {
        v = P::load(row, column, width);
#pragma unroll
        for (int e = 0; e < P::V; e++) v[e] = T(__builtin_fmaf(acc[e], scale, float(v[e])));
    } else {
#pragma unroll
        for (int e = 0; e < P::V; e++) v[e] = T(acc[e] * scale);
    }
    P::store(row, column, width, v);
}

template <int V>
__device__ __forceinline__ void put_partial(float *p, const float (&acc)[V])
{
    typedef float Four __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int e = 0; e < V; e += 4) *reinterpret_cast<Four *>(p + e) = Four{acc[e], acc[e + 1], acc[e + 2], acc[e + 3]};
}

// Sums: bound by reading dout, once the waves are enough: 65536 x 1024 bfloat16 23.4 us (134 MB, 5.8 TB/s), 8192 x 2048 12.7 us (33 MB read, some 5000 rows
// of 4 KB written).  A wave sums one strip of a chunk of sorted tokens: kAhead rows are on their way at a time.  A run of tokens of one id that ends within the chunk
// it began in is finished here; what a chunk has of a run that came from the chunk before, and of one that goes on in the next, is left for join_runs.
constexpr int kAhead = 8;
template <typename T>
__global__ __launch_bounds__(kBlock) void sum_chunks(const EmbedHeader *header, const SortedToken *__restrict__ list,
                                                     const T *__restrict__ dout, int64_t width, uint32_t strips, int32_t chunk, float scale,
                                                     int32_t accumulate, T *__restrict__ dtable, float *__restrict__ partial, int64_t pitch)
{
    using P = Piece<T>;
    const int lane = int(threadIdx.x) & 63;
    const uint32_t item = blockIdx.x * (kBlock / 64) + uint32_t(__builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6));
    const uint32_t at = item / strips, strip = item % strips;
    const int64_t count = header->count, p0 = int64_t(at) * chunk;
    if (p0 >= count) return;
    const int n = int(count - p0 < chunk ? count - p0 : chunk);
    const SortedToken held = lane < n ? list[p0 + lane] : SortedToken{-1, 0};
    const int32_t mine = held.id, from = held.token;
    const int32_t before = p0 > 0 ? list[p0 - 1].id : -1, after = p0 + n < count ? list[p0 + n].id : -1;
    const int64_t column = (int64_t(strip) * 64 + lane) * P::V;
    const bool there = column < width;
    float acc[P::V];
#pragma unroll
    for (int e = 0; e < P::V; e++) acc[e] = 0.f;
    int32_t id = __builtin_amdgcn_readlane(mine, 0);
    bool carried = id == before;
    for (int k0 = 0; k0 < n; k0 += kAhead) {
        typename P::Vec v[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; k++) {
            const int j = k0 + k < n ? k0 + k : n - 1;
            const int64_t token = __builtin_amdgcn_readlane(from, j);
            v[k] = there ? P::load(dout + token * width, column, width) : typename P::Vec(T(0.f));
        }
#pragma unroll
        for (int k = 0; k < kAhead; k++) {
            if (k0 + k >= n) break;
#pragma unroll
            for (int e = 0; e < P::V; e++) acc[e] += float(v[k][e]);
            const bool end = k0 + k + 1 == n;
            const int32_t next = end ? after : __builtin_amdgcn_readlane(mine, (k0 + k + 1) & 63);
            if (next == id && !end) continue;
            const bool goes_on = next == id;
            if (carried || goes_on) put_partial(partial + (int64_t(at) * 2 + (carried ? 0 : 1)) * pitch + column, acc);
            else if (there) finish<T>(acc, scale, accumulate != 0, dtable + int64_t(id) * width, column, width);
            carried = false;
            id = next;
#pragma unroll
            for (int e = 0; e < P::V; e++) acc[e] = 0.f;
        }
    }
}

// Runs that go over the end of the chunk they began in: their parts, in order.  Latency: a launch, whose blocks find out whether they have one, and a few
// rounds of loads; 5 us for 8192 tokens, 8 where a run has 10000 tokens.  2, 4, 8 and 16 waves: 5.4, 5.0, 5.1, 8.0 and 10.3, 8.5, 8.0, 9.1 us.  A block per chunk and strip, whose waves take a share of the
// chunks each.
constexpr int kJoinWaves = 8;
template <typename T>
__global__ __launch_bounds__(64 * kJoinWaves) void join_runs(const EmbedHeader *header, const SortedToken *__restrict__ list, int64_t width,
                                                             uint32_t strips, int32_t chunk, float scale, int32_t accumulate,
                                                             T *__restrict__ dtable, const float *__restrict__ partial, int64_t pitch)
{
    using P = Piece<T>;
    typedef float Four __attribute__((ext_vector_type(4)));
    __shared__ __align__(16) float sums[kJoinWaves][64 * P::V];
    const int lane = int(threadIdx.x) & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
    const int64_t at = blockIdx.x / strips, strip = blockIdx.x % strips;
    const int64_t count = header->count, p0 = at * chunk;
    if (p0 + chunk >= count) return;                     // nothing after this chunk
    const int32_t id = list[p0 + chunk - 1].id;
    if (list[p0 + chunk].id != id || (p0 > 0 && list[p0 - 1].id == id)) return;
    // the last chunk that begins with this id, 64 guesses at a time
    int64_t last = at + 1, end = (count + chunk - 1) / chunk;
    while (end - last > 1) {
        const int64_t step = (end - last + 63) / 64, guess = last + lane * step;
        const int found_here = __popcll(__ballot(guess < end && list[(guess < end ? guess : last) * chunk].id == id)), same = found_here > 0 ? found_here : 1;
        const int64_t found = last + int64_t(same - 1) * step;
        end = found + step < end ? found + step : end;
        last = found;
    }
    const int64_t column = (strip * 64 + lane) * P::V, parts = last - at, each = (parts + kJoinWaves - 1) / kJoinWaves;
    const int64_t to = at + 1 + (wave + 1) * each < last + 1 ? at + 1 + (wave + 1) * each : last + 1;
    float acc[P::V];
    const auto add = [&](const float *p) {
#pragma unroll
        for (int e = 0; e < P::V; e += 4) {
            const Four v = *reinterpret_cast<const Four *>(p + e);
            acc[e] += v[0];
            acc[e + 1] += v[1];
            acc[e + 2] += v[2];
            acc[e + 3] += v[3];
        }
    };
#pragma unroll
    for (int e = 0; e < P::V; e++) acc[e] = 0.f;
    if (wave == 0) add(partial + (at * 2 + 1) * pitch + column);
#pragma unroll 8
    for (int64_t c = at + 1 + wave * each; c < to; c++) add(partial + c * 2 * pitch + column);
    put_partial(&sums[wave][lane * P::V], acc);
    __syncthreads();
    if (wave != 0 || column >= width) return;
#pragma unroll
    for (int e = 0; e < P::V; e++) acc[e] = 0.f;
    for (int w = 0; w < kJoinWaves; w++) add(&sums[w][lane * P::V]);
    finish<T>(acc, scale, accumulate != 0, dtable + int64_t(id) * width, column, width);
}

// Few tokens: no sort.  Every wave holds all ids, two a lane, and finds the tokens of a row by votes.  A wave takes a strip of `each` rows of the table,
// one after another, or (accumulate) that of one token's row, if it is the first token of its id.  Bound by writing zeros, or by its launch: 100 x 2048 of 50257
// bfloat16 38 us (5.5 TB/s; 300 tokens, sorted, 46), 100 x 768 of 5000 binary32 7.3 (13 to 15 sorted).
constexpr int kFewTokens = 128;
template <typename T>
__global__ __launch_bounds__(kBlock) void few_rows(const int64_t *__restrict__ ids, const T *__restrict__ dout, int32_t tokens, int64_t ignore,
                                                   int64_t vocab, int64_t width, uint32_t strips, float scale, int32_t accumulate,
                                                   T *__restrict__ dtable, int32_t each)
{
    using P = Piece<T>;
    const int lane = int(threadIdx.x) & 63;
    const int64_t item = int64_t(blockIdx.x) * (kBlock / 64) + __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6), at = item / strips;
    const int64_t column = (item % strips * 64 + lane) * P::V;
    const auto id_of = [&](int32_t token) {
        const int64_t id = token < tokens ? ids[token] : -1;
        return id >= 0 && id < vocab && id != ignore ? int32_t(id) : -1;
    };
    const int32_t low = id_of(lane), high = id_of(64 + lane);
    const auto sum = [&](uint64_t first, uint64_t second, int32_t id) {
        float acc[P::V];
#pragma unroll
        for (int e = 0; e < P::V; e++) acc[e] = 0.f;
        while (first | second) {
            typename P::Vec v[kAhead];
            int n = 0;
#pragma unroll
            for (int k = 0; k < kAhead; k++) {
                v[k] = typename P::Vec(T(0.f));
                if (!(first | second)) continue;
                const int64_t token = first ? __builtin_ctzll(first) : 64 + __builtin_ctzll(second);
                if (first) first &= first - 1;
                else second &= second - 1;
                if (column < width) v[k] = P::load(dout + token * width, column, width);
                n = k + 1;
            }
#pragma unroll
            for (int k = 0; k < kAhead; k++) {
                if (k >= n) break;
#pragma unroll
                for (int e = 0; e < P::V; e++) acc[e] += float(v[k][e]);
            }
        }
        if (column < width) finish<T>(acc, scale, accumulate != 0, dtable + int64_t(id) * width, column, width);
    };
    if (accumulate) {
        if (at >= tokens) return;
        const int32_t id = at < 64 ? __builtin_amdgcn_readlane(low, int(at)) : __builtin_amdgcn_readlane(high, int(at) - 64);
        const uint64_t first = __ballot(low == id), second = __ballot(high == id);
        if (id < 0 || (at < 64 ? first & ((uint64_t(1) << at) - 1) : first | (second & ((uint64_t(1) << (at - 64)) - 1)))) return;
        sum(first, second, id);
        return;
    }
    for (int64_t row = at * each; row < (at + 1) * each && row < vocab; row++) {
        const uint64_t first = __ballot(low == int32_t(row)), second = __ballot(high == int32_t(row));
        if (first | second) sum(first, second, int32_t(row));
        else if (column < width) P::store(dtable + row * width, column, width, typename P::Vec(T(0.f)));
    }
}

// ---------------------------------------------------------------- launches

struct Launches {
    hipStream_t stream;
    hipError_t error = hipSuccess;           // of the first launch that was refused
    void launched()
    {
        const hipError_t e = hipGetLastError();
        if (error == hipSuccess) error = e;
    }
};

template <typename T>
hipError_t look_up_all(const void *table, const int64_t *ids, int64_t tokens, int64_t width, int64_t vocab, int64_t ignore, float scale, void *out,
                       hipStream_t stream)
{
    Launches l{stream};
    const int64_t strips = (width + 64 * Piece<T>::V - 1) / (64 * Piece<T>::V);
    const auto go = [&](auto each) {
        constexpr int EACH = decltype(each)::value;
        const int64_t parts = (strips + EACH - 1) / EACH;
        look_up<T, EACH><<<dim3(uint32_t((tokens * parts + kBlock / 64 - 1) / (kBlock / 64))), kBlock, 0, stream>>>(
            static_cast<const T *>(table), ids, tokens, width, vocab, ignore, scale, uint32_t(parts), static_cast<T *>(out));
        l.launched();
    };
    if (strips >= 4 && tokens * strips >= 8192) go(std::integral_constant<int, 4>());
    else if (strips >= 2 && tokens * strips >= 4096) go(std::integral_constant<int, 2>());
    else go(std::integral_constant<int, 1>());
    return l.error;
}

template <typename T>
hipError_t gradient(const EmbedLayout &l, const void *dout, const int64_t *ids, int64_t ignore, float scale, bool accumulate, void *dtable,
                    unsigned char *ws, hipStream_t stream)
{
    Launches g{stream};
    if (l.tokens && l.tokens <= kFewTokens) {
        // (one row a wave while the chip holds twice as many waves; a launch has fewer than 2^32 threads)
        const int64_t each = l.vocab * l.strips <= 16384 ? 1 : l.vocab < int64_t(1) << 26 ? 4 : 16;
        const int64_t items = (accumulate ? l.tokens : (l.vocab + each - 1) / each) * l.strips;
        few_rows<T><<<dim3(uint32_t((items + kBlock / 64 - 1) / (kBlock / 64))), kBlock, 0, stream>>>(
            ids, static_cast<const T *>(dout), int32_t(l.tokens), ignore, l.vocab, l.width, uint32_t(l.strips), scale, accumulate,
            static_cast<T *>(dtable), int32_t(each));
        g.launched();
        return g.error;
    }
    const auto at = [ws](size_t offset) { return reinterpret_cast<SortedToken *>(ws + offset); };
    EmbedHeader *header = reinterpret_cast<EmbedHeader *>(ws);
    SortedToken *const list = at(l.list[0]);
    const Parts parts{at(l.part), reinterpret_cast<uint32_t *>(ws + l.starts), uint32_t((l.tokens + kEmbedParts - 1) / kEmbedParts), l.bits};
    const int64_t bytes = l.vocab * l.width * int64_t(sizeof(T)), fills = accumulate ? 0 : (bytes + kFillBytes - 1) / kFillBytes;
    const uint32_t sorts = l.tokens ? uint32_t(l.blocks) : 0, grid = sorts + uint32_t(fills);
    if (l.parts) {
        sort_parts<<<dim3(kEmbedParts), kSortThreads, 0, stream>>>(ids, uint32_t(l.tokens), ignore, l.vocab, l.blocks, parts);
        g.launched();
    }
    const auto sort = [&](auto fill, auto in_parts) {
        sort_tokens<decltype(fill)::value, decltype(in_parts)::value><<<dim3(grid), kSortThreads, 0, stream>>>(
            ids, uint32_t(l.tokens), ignore, l.vocab, l.share, l.bits, sorts, header, list, at(l.list[1]), parts, static_cast<unsigned char *>(dtable), bytes);
        g.launched();
    };
    if (grid) {
        const std::true_type yes;
        const std::false_type no;
        if (l.parts) fills ? sort(yes, yes) : sort(no, yes);
        else fills ? sort(yes, no) : sort(no, no);
    }
    if (!l.tokens) return g.error;
    float *partial = reinterpret_cast<float *>(ws + l.partial);
    const int64_t items = l.chunks * l.strips;
    sum_chunks<T><<<dim3(uint32_t((items + kBlock / 64 - 1) / (kBlock / 64))), kBlock, 0, stream>>>(
        header, list, static_cast<const T *>(dout), l.width, uint32_t(l.strips), l.chunk, scale, accumulate,
        static_cast<T *>(dtable), partial, l.pitch);
    g.launched();
    if (l.chunks > 1) {
        join_runs<T><<<dim3(uint32_t((l.chunks - 1) * l.strips)), 64 * kJoinWaves, 0, stream>>>(
            header, list, l.width, uint32_t(l.strips), l.chunk, scale, accumulate, static_cast<T *>(dtable), partial, l.pitch);
        g.launched();
    }
    return g.error;
}

}  // namespace

int launch_embed(const void *table, const int64_t *ids, int64_t tokens, int64_t width, int64_t vocab, int dt, int64_t ignore, float scale,
                 void *out, void *stream)
{
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (dt == CGX_F32) return look_up_all<float>(table, ids, tokens, width, vocab, ignore, scale, out, s);
    if (dt == CGX_F16) return look_up_all<_Float16>(table, ids, tokens, width, vocab, ignore, scale, out, s);
    return look_up_all<__bf16>(table, ids, tokens, width, vocab, ignore, scale, out, s);
}

int launch_embed_grad(const EmbedLayout &l, const void *dout, const int64_t *ids, int64_t ignore, float scale, bool accumulate, void *dtable,
                      unsigned char *workspace, void *stream)
{
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (l.dt == CGX_F32) return gradient<float>(l, dout, ids, ignore, scale, accumulate, dtable, workspace, s);
    if (l.dt == CGX_F16) return gradient<_Float16>(l, dout, ids, ignore, scale, accumulate, dtable, workspace, s);
    return gradient<__bf16>(l, dout, ids, ignore, scale, accumulate, dtable, workspace, s);
}

}  // namespace cgx
