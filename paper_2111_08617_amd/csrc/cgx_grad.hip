// Global norm of a list of gradient tensors, and their clipping by it: kernels and launches.
//
// Both are streaming kernels, bound by memory: the norm reads every element once, the clipping reads and writes it once, and a
// byte of it costs less than one vector instruction.  What sets their time besides is the number of launches, so the
// table of tensors travels in the kernels' arguments (nothing is copied to the device ahead of a launch) and one launch serves
// as many tensors as the arguments hold.
#include "cgx_grad.h"

#include <type_traits>

namespace cgx {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kBlock = 256;
constexpr int kItem = 8192;                          // elements that a block takes at a time
constexpr int kEntries = 160;                        // of 24 bytes: a launch's arguments stay under 4 KB
constexpr int kClipBlocks = 4096;

struct Entry {
    const void *src;
    void *dst;               // clipping
    uint32_t first;          // number of the tensor's first item
    uint32_t last;           // elements of its last item, and its type in bits 30 and 31
};
struct Group {
    Entry entry[kEntries];
};

// Which tensor an item belongs to: each lane keeps the first items of a few entries, and votes.
struct Finder {
    static constexpr int kEach = (kEntries + 63) / 64;
    uint32_t first[kEach];
    __device__ __forceinline__ Finder(const Group &group, int32_t entries)
    {
        const int lane = int(threadIdx.x) & 63;
#pragma unroll
        for (int k = 0; k < kEach; k++) first[k] = k * 64 + lane < entries ? group.entry[k * 64 + lane].first : 0xffffffffu;
    }
    __device__ __forceinline__ int operator()(uint32_t item) const
    {
        int at = -1;
#pragma unroll
        for (int k = 0; k < kEach; k++) at += __popcll(__ballot(first[k] <= item));
        return __builtin_amdgcn_readfirstlane(at);
    }
};

// Elements of the item of an entry (the next entry's first item, or the launch's end, bounds it).
__device__ __forceinline__ uint32_t elements_of(const Group &group, int at, int32_t entries, uint32_t items, uint32_t item)
{
    const uint32_t end = at + 1 < entries ? group.entry[at + 1].first : items;
    return item + 1 == end ? group.entry[at].last & 0x3fffffffu : uint32_t(kItem);
}

// Eight elements as stored, and widened.  Tensors start at any element: the loads are aligned like one.
template <int DT>
struct Stored;
template <>
struct Stored<CGX_F32> {
    typedef float Element;
    typedef f32x8 Raw;
    static __device__ __forceinline__ f32x8 widen(const Raw &r) { return r; }
};
template <>
struct Stored<CGX_F16> {
    typedef _Float16 Element;
    typedef f16x8 Raw;
    static __device__ __forceinline__ f32x8 widen(const Raw &r) { return __builtin_convertvector(r, f32x8); }
};
template <>
struct Stored<CGX_BF16> {
    typedef __bf16 Element;
    typedef bf16x8 Raw;
    static __device__ __forceinline__ f32x8 widen(const Raw &r) { return __builtin_convertvector(r, f32x8); }
};
template <int DT>
struct Anywhere {
    typedef typename Stored<DT>::Raw Raw __attribute__((aligned(sizeof(typename Stored<DT>::Element))));
};

constexpr int kVectors = kItem / 8 / kBlock;         // vectors of eight elements that a thread takes of a whole item

template <int DT>
__device__ __forceinline__ double squares(const typename Stored<DT>::Element *p, uint32_t n)
{
    using Raw = typename Anywhere<DT>::Raw;
    const Raw *v = reinterpret_cast<const Raw *>(p);
    const uint32_t vectors = n / 8;
    f32x8 x[kVectors];
#pragma unroll
    for (int k = 0; k < kVectors; k++) {
        const uint32_t at = k * kBlock + threadIdx.x;
        x[k] = f32x8{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (at < vectors) {
            const typename Stored<DT>::Raw stored = v[at];
            x[k] = Stored<DT>::widen(stored);
        }
    }
    double sum = 0.0;
#pragma unroll
    for (int k = 0; k < kVectors; k++)
#pragma unroll
        for (int e = 0; e < 8; e++) sum += double(x[k][e]) * double(x[k][e]);
    const uint32_t at = vectors * 8 + threadIdx.x;
    if (at < n) sum += double(float(p[at])) * double(float(p[at]));
    return sum;
}

// Sums over a block, in a fixed order; the result is thread 0's.
__device__ __forceinline__ double block_sum(double v, double *waves)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = v;
    __syncthreads();
    double sum = 0.0;
    for (int w = 0; w < int(blockDim.x) / 64; w++) sum += waves[w];
    return sum;
}

// A block's share of the squares: items block, block + grid, ... of the launch.  Squares of binary32 values are exact in binary64,
// so nothing overflows and only the additions round; no atomics, so a norm is the same bits every time.
__global__ __launch_bounds__(kBlock) void norm_items(Group group, int32_t entries, uint32_t items, double *partial, int32_t add)
{
    __shared__ double waves[kBlock / 64];
    const Finder find(group, entries);
    double sum = 0.0;
    for (uint32_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int at = find(item);
        const Entry &e = group.entry[at];
        const uint32_t n = elements_of(group, at, entries, items, item);
        const int64_t from = int64_t(item - e.first) * kItem;
        const uint32_t dt = e.last >> 30;
        if (dt == CGX_F32) sum += squares<CGX_F32>(static_cast<const float *>(e.src) + from, n);
        else if (dt == CGX_F16) sum += squares<CGX_F16>(static_cast<const _Float16 *>(e.src) + from, n);
        else sum += squares<CGX_BF16>(static_cast<const __bf16 *>(e.src) + from, n);
    }
    sum = block_sum(sum, waves);
    if (threadIdx.x == 0) partial[blockIdx.x] = add ? partial[blockIdx.x] + sum : sum;
}

__global__ __launch_bounds__(1024) void norm_join(const double *__restrict__ partial, int32_t count, float *norm)
{
    __shared__ double waves[1024 / 64];
    double sum = 0.0;
    for (int32_t k = int32_t(threadIdx.x); k < count; k += 1024) sum += partial[k];
    sum = block_sum(sum, waves);
    if (threadIdx.x == 0) *norm = float(sqrt(sum));
}

template <int DT, int OUT>
__device__ __forceinline__ void scale_item(const void *src, void *dst, int64_t from, uint32_t n, float factor)
{
    using Element = typename Stored<DT>::Element;
    using Result = typename Stored<OUT>::Element;
    using Raw = typename Anywhere<DT>::Raw;
    using Out = typename Anywhere<OUT>::Raw;
    const Element *p = static_cast<const Element *>(src) + from;
    Result *q = static_cast<Result *>(dst) + from;
    const uint32_t vectors = n / 8;
    Raw x[kVectors];
#pragma unroll
    for (int k = 0; k < kVectors; k++) {
        const uint32_t at = k * kBlock + threadIdx.x;
        if (at < vectors) x[k] = reinterpret_cast<const Raw *>(p)[at];
    }
#pragma unroll
    for (int k = 0; k < kVectors; k++) {
        const uint32_t at = k * kBlock + threadIdx.x;
        if (at < vectors) {
            const typename Stored<DT>::Raw stored = x[k];
            f32x8 f = Stored<DT>::widen(stored);
#pragma unroll
            for (int e = 0; e < 8; e++) f[e] *= factor;
            reinterpret_cast<Out *>(q)[at] = __builtin_convertvector(f, typename Stored<OUT>::Raw);
        }
    }
    const uint32_t at = vectors * 8 + threadIdx.x;
    if (at < n) q[at] = Result(float(p[at]) * factor);
}

// x * factor, in place (OUT < 0: each tensor in its own type) or into the fused buffer.
template <int OUT>
__global__ __launch_bounds__(kBlock) void clip_items(Group group, int32_t entries, uint32_t items, const float *norm, float max_norm)
{
    const float size = *norm;
    const float factor = size > max_norm ? max_norm / size : size == size ? 1.f : size;
    if (OUT < 0 && factor == 1.f) return;
    const Finder find(group, entries);
    for (uint32_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int at = find(item);
        const Entry &e = group.entry[at];
        const uint32_t n = elements_of(group, at, entries, items, item);
        const int64_t from = int64_t(item - e.first) * kItem;
        const uint32_t dt = e.last >> 30;
        if (dt == CGX_F32) scale_item<CGX_F32, OUT < 0 ? int(CGX_F32) : OUT>(e.src, e.dst, from, n, factor);
        else if (dt == CGX_F16) scale_item<CGX_F16, OUT < 0 ? int(CGX_F16) : OUT>(e.src, e.dst, from, n, factor);
        else scale_item<CGX_BF16, OUT < 0 ? int(CGX_BF16) : OUT>(e.src, e.dst, from, n, factor);
    }
}

int64_t items_of(const cgx_tensor &t) { return (t.n + kItem - 1) / kItem; }

// The list in groups that a launch's arguments hold; launch(group, entries, items) for each.  A group has fewer than 2^31 items.
template <typename Launch>
hipError_t each_group(const cgx_tensor *tensors, int32_t count, unsigned char *out, int out_size, const Launch &launch)
{
    Group group;
    int32_t entries = 0;
    int64_t items = 0;
    hipError_t e = hipSuccess;
    const auto flush = [&] {
        if (entries) launch(group, entries, uint32_t(items));
        if (entries) e = hipGetLastError();
        entries = 0;
        items = 0;
    };
    for (int32_t k = 0; k < count && e == hipSuccess; k++) {
        const cgx_tensor &t = tensors[k];
        if (t.n == 0) continue;
        if (entries == kEntries || items + items_of(t) >= (int64_t(1) << 31)) flush();
        const int64_t last = t.n - (items_of(t) - 1) * kItem;
        group.entry[entries++] = Entry{t.data, out ? out : t.data, uint32_t(items), uint32_t(last) | uint32_t(t.dt) << 30};
        items += items_of(t);
        if (out) out += t.n * out_size;
    }
    if (e == hipSuccess) flush();
    return e;
}

}  // namespace

hipError_t launch_grad_norm(const cgx_tensor *tensors, int32_t count, float *norm, double *partial, hipStream_t stream)
{
    // every launch runs the same blocks, so that each slot is written by the first one
    int64_t items = 0;
    for (int32_t k = 0; k < count; k++) items += items_of(tensors[k]);
    const int32_t blocks = int32_t(items < kNormSlots ? items : kNormSlots);
    int32_t done = 0;
    const hipError_t e = each_group(tensors, count, nullptr, 0, [&](const Group &group, int32_t entries, uint32_t n) {
        norm_items<<<dim3(uint32_t(blocks)), kBlock, 0, stream>>>(group, entries, n, partial, done++ > 0);
    });
    if (e != hipSuccess) return e;
    norm_join<<<1, 1024, 0, stream>>>(partial, blocks, norm);
    return hipGetLastError();
}

hipError_t launch_grad_clip(const cgx_tensor *tensors, int32_t count, const float *norm, float max_norm, void *out, int out_dt,
                            hipStream_t stream)
{
    return each_group(tensors, count, static_cast<unsigned char *>(out), out_dt == CGX_F32 ? 4 : 2,
                      [&](const Group &group, int32_t entries, uint32_t n) {
                          const dim3 grid(n < uint32_t(kClipBlocks) ? n : uint32_t(kClipBlocks));
                          if (!out) clip_items<-1><<<grid, kBlock, 0, stream>>>(group, entries, n, norm, max_norm);
                          else if (out_dt == CGX_F32) clip_items<CGX_F32><<<grid, kBlock, 0, stream>>>(group, entries, n, norm, max_norm);
                          else if (out_dt == CGX_F16) clip_items<CGX_F16><<<grid, kBlock, 0, stream>>>(group, entries, n, norm, max_norm);
                          else clip_items<CGX_BF16><<<grid, kBlock, 0, stream>>>(group, entries, n, norm, max_norm);
                      });
}

}  // namespace cgx
