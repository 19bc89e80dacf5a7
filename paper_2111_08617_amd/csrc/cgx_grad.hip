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

constexpr int kBlock = 256;
// Elements that a block takes at a time.  (1.3 G bfloat16 gradients clipped into binary32, norm included, in us: 1744 with 4096, 1793
// with 8192, 1800 with 2048; a grid of 4096 blocks that walks them takes 5 % more than a block each.)
constexpr int kItem = 4096;
constexpr int kEntries = 240;                        // of 16 bytes: a launch's arguments stay under 4 KB
constexpr int kClipBlocks = 1 << 23;                 // (a grid has fewer than 2^32 threads)

struct Entry {
    const void *data;
    uint32_t first;          // number of the tensor's first item
    uint32_t lack;           // elements that the last items of the tensors before it lack, in all; its type in bits 30 and 31
};
struct Group {
    Entry entry[kEntries];
    int32_t entries;
    uint32_t items, lack;    // of the launch: where the last tensor ends
};

// Which tensor an item belongs to: each lane keeps the first items of a few entries, and votes.
struct Finder {
    static constexpr int kEach = (kEntries + 63) / 64;
    uint32_t first[kEach];
    __device__ __forceinline__ explicit Finder(const Group &group)
    {
        const int lane = int(threadIdx.x) & 63;
#pragma unroll
        for (int k = 0; k < kEach; k++) first[k] = k * 64 + lane < group.entries ? group.entry[k * 64 + lane].first : 0xffffffffu;
    }
    __device__ __forceinline__ int operator()(uint32_t item) const
    {
        int at = -1;
#pragma unroll
        for (int k = 0; k < kEach; k++) at += __popcll(__ballot(first[k] <= item));
        return __builtin_amdgcn_readfirstlane(at);
    }
};

// An item: where it lies, in its tensor and in all tensors of the launch one after another, and how long it is.
struct Item {
    const void *data;
    int64_t from, place;
    uint32_t n;
    int dt;
};
__device__ __forceinline__ Item item_of(const Group &group, const Finder &find, uint32_t item)
{
    const int at = find(item);
    const Entry &e = group.entry[at];
    const bool last = at + 1 == group.entries;
    const uint32_t lack = e.lack & 0x3fffffffu, end = last ? group.items : group.entry[at + 1].first;
    const uint32_t after = last ? group.lack : group.entry[at + 1].lack & 0x3fffffffu;
    return {e.data, int64_t(item - e.first) * kItem, int64_t(item) * kItem - lack, item + 1 == end ? uint32_t(kItem) - (after - lack) : uint32_t(kItem),
            int(e.lack >> 30)};
}

// V elements as stored, and their values.  A lane's V elements are at most 16 bytes on either side, so that every load and store
// instruction of a wave covers consecutive addresses.  Tensors start at any element: accesses are aligned like one.
template <int DT>
struct Stored;
template <>
struct Stored<CGX_F32> {
    typedef float Element;
};
template <>
struct Stored<CGX_F16> {
    typedef _Float16 Element;
};
template <>
struct Stored<CGX_BF16> {
    typedef __bf16 Element;
};
template <int DT, int V>
struct Vector {
    typedef typename Stored<DT>::Element Element;
    typedef Element Value __attribute__((ext_vector_type(V)));
    typedef Value Anywhere __attribute__((aligned(sizeof(Element))));
};
template <int DT>
constexpr int per_lane = 16 / int(sizeof(typename Stored<DT>::Element));

// STREAM: the tensors are larger than the memory-side cache, and nothing of them will be found there: loads do not fill the caches.
template <int DT, bool STREAM>
__device__ __forceinline__ double squares(const typename Stored<DT>::Element *p, uint32_t n)
{
    constexpr int V = per_lane<DT>, kEach = kItem / V / kBlock;
    using Value = typename Vector<DT, V>::Value;
    const auto *v = reinterpret_cast<const typename Vector<DT, V>::Anywhere *>(p);
    const uint32_t vectors = n / V;
    Value x[kEach];
#pragma unroll
    for (int k = 0; k < kEach; k++) {
        const uint32_t at = k * kBlock + threadIdx.x;
        x[k] = Value(0.f);
        if (at < vectors) x[k] = STREAM ? __builtin_nontemporal_load(v + at) : v[at];
    }
    double sum = 0.0;
#pragma unroll
    for (int k = 0; k < kEach; k++)
#pragma unroll
        for (int e = 0; e < V; e++) sum += double(float(x[k][e])) * double(float(x[k][e]));
    const uint32_t at = vectors * V + threadIdx.x;
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
// 2.2 GB of bfloat16: 330 us (6.7 TB/s); 102 MB of binary32 17 us (6 TB/s); some tens of small tensors 3.5 us.
template <bool STREAM>
__global__ __launch_bounds__(kBlock) void norm_items(Group group, double *partial, int32_t add)
{
    __shared__ double waves[kBlock / 64];
    const Finder find(group);
    double sum = 0.0;
    for (uint32_t item = blockIdx.x; item < group.items; item += gridDim.x) {
        const Item i = item_of(group, find, item);
        if (i.dt == CGX_F32) sum += squares<CGX_F32, STREAM>(static_cast<const float *>(i.data) + i.from, i.n);
        else if (i.dt == CGX_F16) sum += squares<CGX_F16, STREAM>(static_cast<const _Float16 *>(i.data) + i.from, i.n);
        else sum += squares<CGX_BF16, STREAM>(static_cast<const __bf16 *>(i.data) + i.from, i.n);
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

template <int DT, int OUT, bool STREAM>
__device__ __forceinline__ void scale_item(const void *src, int64_t from, void *dst, int64_t to, uint32_t n, float factor)
{
    constexpr int V = per_lane<DT> < per_lane<OUT> ? per_lane<DT> : per_lane<OUT>, kEach = kItem / V / kBlock;
    using Value = typename Vector<DT, V>::Value;
    using Result = typename Stored<OUT>::Element;
    const typename Stored<DT>::Element *p = static_cast<const typename Stored<DT>::Element *>(src) + from;
    Result *q = static_cast<Result *>(dst) + to;
    const auto *v = reinterpret_cast<const typename Vector<DT, V>::Anywhere *>(p);
    auto *w = reinterpret_cast<typename Vector<OUT, V>::Anywhere *>(q);
    const uint32_t vectors = n / V;
    Value x[kEach];
#pragma unroll
    for (int k = 0; k < kEach; k++) {
        const uint32_t at = k * kBlock + threadIdx.x;
        if (at < vectors) x[k] = v[at];
    }
#pragma unroll
    for (int k = 0; k < kEach; k++) {
        const uint32_t at = k * kBlock + threadIdx.x;
        if (at < vectors) {
            typename Vector<OUT, V>::Value y;
#pragma unroll
            for (int e = 0; e < V; e++) y[e] = Result(float(x[k][e]) * factor);
            if (STREAM) __builtin_nontemporal_store(y, w + at);
            else w[at] = y;
        }
    }
    const uint32_t at = vectors * V + threadIdx.x;
    if (at < n) q[at] = Result(float(p[at]) * factor);
}

// x * factor, in place (OUT < 0: each tensor in its own type) or into the fused buffer.  factor = min(1, max_norm / norm) in binary32;
// the product is rounded once, to the result's type.  2.2 GB of bfloat16 into 4.4 GB of binary32: 1120 us (5.9 TB/s; a copy of 4 GB
// by the library 4.75); 102 MB of binary32, which the norm has left in the memory-side cache, 31 us (6.6 TB/s).  In place, 5.3 GB of binary32:
// 1890 us (5.6 TB/s).
template <int OUT, bool STREAM>
__global__ __launch_bounds__(kBlock) void clip_items(Group group, const float *norm, float max_norm, void *out)
{
    const float size = *norm;
    const float factor = size > max_norm ? max_norm / size : size == size ? 1.f : size;
    if (OUT < 0 && factor == 1.f) return;
    const Finder find(group);
    for (uint32_t item = blockIdx.x; item < group.items; item += gridDim.x) {
        const Item i = item_of(group, find, item);
        void *const dst = OUT < 0 ? const_cast<void *>(i.data) : out;
        const int64_t to = OUT < 0 ? i.from : i.place;
        if (i.dt == CGX_F32) scale_item<CGX_F32, OUT < 0 ? int(CGX_F32) : OUT, STREAM>(i.data, i.from, dst, to, i.n, factor);
        else if (i.dt == CGX_F16) scale_item<CGX_F16, OUT < 0 ? int(CGX_F16) : OUT, STREAM>(i.data, i.from, dst, to, i.n, factor);
        else scale_item<CGX_BF16, OUT < 0 ? int(CGX_BF16) : OUT, STREAM>(i.data, i.from, dst, to, i.n, factor);
    }
}

int64_t size_of(int dt) { return dt == CGX_F32 ? 4 : 2; }
int64_t items_of(const cgx_tensor &t) { return (t.n + kItem - 1) / kItem; }

// The list in groups that a launch's arguments hold; launch(group, elements in the groups before it) for each.  A group has fewer than
// 2^31 items.
template <typename Launch>
hipError_t each_group(const cgx_tensor *tensors, int32_t count, const Launch &launch)
{
    static_assert(sizeof(Group) + 32 <= 4096 && kEntries * kItem < (1 << 30), "see Entry");
    Group group;
    int64_t items = 0, lack = 0, done = 0;
    hipError_t e = hipSuccess;
    group.entries = 0;
    const auto flush = [&] {
        if (!group.entries) return;
        group.items = uint32_t(items);
        group.lack = uint32_t(lack);
        launch(group, done);
        e = hipGetLastError();
        done += items * kItem - lack;
        items = lack = group.entries = 0;
    };
    for (int32_t k = 0; k < count && e == hipSuccess; k++) {
        const cgx_tensor &t = tensors[k];
        if (t.n == 0) continue;
        if (group.entries == kEntries || items + items_of(t) >= (int64_t(1) << 31)) flush();
        group.entry[group.entries++] = Entry{t.data, uint32_t(items), uint32_t(lack) | uint32_t(t.dt) << 30};
        items += items_of(t);
        lack += items_of(t) * kItem - t.n;
    }
    if (e == hipSuccess) flush();
    return e;
}

}  // namespace

hipError_t launch_grad_norm(const cgx_tensor *tensors, int32_t count, float *norm, double *partial, hipStream_t stream)
{
    // every launch runs the same blocks, so that each slot is written by the first one
    int64_t items = 0, bytes = 0;
    for (int32_t k = 0; k < count; k++) {
        items += items_of(tensors[k]);
        bytes += tensors[k].n * size_of(tensors[k].dt);
    }
    // the clipping that follows finds what fits the 256 MB memory-side cache there (102 MB clipped: 51.5 us, 54.6 with streaming loads);
    // beyond that streaming loads are faster (710 MB: 128 and 119 us)
    const bool stream_loads = bytes > (int64_t(256) << 20);
    const int32_t blocks = int32_t(items < kNormSlots ? items : kNormSlots);
    int32_t done = 0;
    const hipError_t e = each_group(tensors, count, [&](const Group &group, int64_t) {
        if (stream_loads) norm_items<true><<<dim3(uint32_t(blocks)), kBlock, 0, stream>>>(group, partial, done++ > 0);
        else norm_items<false><<<dim3(uint32_t(blocks)), kBlock, 0, stream>>>(group, partial, done++ > 0);
    });
    if (e != hipSuccess) return e;
    norm_join<<<1, 1024, 0, stream>>>(partial, blocks, norm);
    return hipGetLastError();
}

hipError_t launch_grad_clip(const cgx_tensor *tensors, int32_t count, const float *norm, float max_norm, void *out, int out_dt,
                            hipStream_t stream)
{
    int64_t bytes = 0;
    for (int32_t k = 0; k < count; k++) bytes += tensors[k].n * (out ? size_of(out_dt) : size_of(tensors[k].dt));
    // results that the memory-side cache holds for the quantizer stay there; larger ones are streamed (5.3 GB: 1813 and 1791 us)
    const bool streams = bytes > (int64_t(128) << 20);
    return each_group(tensors, count, [&](const Group &group, int64_t before) {
        void *const to = out ? static_cast<unsigned char *>(out) + before * size_of(out_dt) : nullptr;
        const auto launch = [&](auto kernel) {
            const dim3 grid(group.items < uint32_t(kClipBlocks) ? group.items : uint32_t(kClipBlocks));
            kernel<<<grid, kBlock, 0, stream>>>(group, norm, max_norm, to);
        };
        if (!out) launch(streams ? clip_items<-1, true> : clip_items<-1, false>);
        else if (out_dt == CGX_F32) launch(streams ? clip_items<CGX_F32, true> : clip_items<CGX_F32, false>);
        else if (out_dt == CGX_F16) launch(streams ? clip_items<CGX_F16, true> : clip_items<CGX_F16, false>);
        else launch(streams ? clip_items<CGX_BF16, true> : clip_items<CGX_BF16, false>);
    });
}

}  // namespace cgx
