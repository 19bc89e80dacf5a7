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
    for (int k = lane; k < t.entries; k += 64) {
        const int64_t id = t.ids[first + k];
        if (id == t.ignore) continue;
        const float x = t.logit(first + k) * t.inverse;
        wrong |= id < 0 || id >= t.vocab || !(x < __builtin_inff());
        r.top = fmaxf(r.top, x);
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) r.top = fmaxf(r.top, __shfl_xor(r.top, d, 64));
    r.wrong = __ballot(wrong) != 0;
    if (r.top == -__builtin_inff()) return r;
    for (int k = lane; k < t.entries; k += 64)
        if (t.ids[first + k] != t.ignore) r.sum += expf(t.logit(first + k) * t.inverse - r.top);
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) r.sum += __shfl_xor(r.sum, d, 64);
    return r;
}

// Which tokens take part: a wave per token.
__global__ __launch_bounds__(256) void mark_tokens(Teacher teacher, int64_t tokens, int64_t *__restrict__ mark)
{
    const int lane = int(threadIdx.x) & 63;
    const int64_t token = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (token >= tokens) return;
    const TeacherRow r = teacher_row(teacher, token, lane);
    if (lane == 0) mark[token] = r.wrong ? kWrong : r.takes_part() ? kTakesPart : kNoPart;
}

// 16 bytes of a row that starts at any element, as binary32.
template <typename T>
struct Slice {
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

// Joins the parts of a token's softmax, takes the student's logits at the teacher's entries (a wave per entry, four at a time), and the divergence.
// A block of WAVES waves per token.
constexpr int kDots = 4;
template <typename T, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void join_divergence(Teacher teacher, const int32_t *__restrict__ place, int64_t parts, int64_t pitch,
                                                              const float2 *__restrict__ stats, const T *__restrict__ hidden,
                                                              const T *__restrict__ weight, int64_t width, float *__restrict__ loss,
                                                              float *__restrict__ lse, float *__restrict__ picked)
{
    __shared__ float sums[WAVES];
    const int tid = int(threadIdx.x), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t token = blockIdx.x;
    const TeacherRow row = teacher_row(teacher, token, lane);
    const int64_t first = token * teacher.entries;
    if (!row.takes_part()) {                             // (the same in all waves)
        for (int k = tid; k < teacher.entries; k += 64 * WAVES) picked[first + k] = 0.f;
        if (tid == 0) loss[token] = lse[token] = 0.f;
        return;
    }
    const float total = log_sum<WAVES>(stats + (place ? int64_t(place[token]) : token) * pitch, parts, tid);
    const float log_mass = row.top + logf(row.sum);
    const T *const x = hidden + token * width;
    float sum = 0.f;
    for (int k0 = wave * kDots; k0 < teacher.entries; k0 += WAVES * kDots) {
        int64_t id[kDots];
        bool inside[kDots];
        float dot[kDots];
#pragma unroll
        for (int k = 0; k < kDots; k++) {
            id[k] = k0 + k < teacher.entries ? teacher.ids[first + k0 + k] : teacher.ignore;
            inside[k] = id[k] != teacher.ignore && id[k] >= 0 && id[k] < teacher.vocab;
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
            if (k0 + k >= teacher.entries) continue;
            const bool marked = id[k] == teacher.ignore;
            if (lane == 0) picked[first + k0 + k] = marked ? 0.f : inside[k] ? dot[k] : __builtin_nanf("");
            if (marked) continue;
            const float scaled = teacher.logit(first + k0 + k) * teacher.inverse, q = row.share(scaled);
            if (q > 0.f) sum += q * (scaled - log_mass + total - dot[k] * teacher.inverse);
        }
    }
    if (lane == 0) sums[wave] = sum;
    __syncthreads();
    if (tid != 0) return;
    sum = 0.f;
    for (int w = 0; w < WAVES; w++) sum += sums[w];
    lse[token] = total;
    loss[token] = row.wrong ? __builtin_nanf("") : sum;
}

// d at the teacher's entries within a piece of the vocabulary, in its units: a wave per token.  An id that comes several times in a row has the sum of
// its shares, written by the first of them.
constexpr int kEntryWaves = 4;
template <typename T>
__global__ __launch_bounds__(64 * kEntryWaves) void delta_entries(Teacher teacher, const int32_t *__restrict__ place, int64_t tokens,
                                                                  const float *__restrict__ lse, const float *__restrict__ factor,
                                                                  const float *__restrict__ picked, int64_t from, int64_t columns,
                                                                  T *__restrict__ delta, int64_t piece)
{
    __shared__ int32_t ids[kEntryWaves][kMostEntries];
    __shared__ float shares[kEntryWaves][kMostEntries];
    const int lane = int(threadIdx.x) & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
    const int64_t token = int64_t(blockIdx.x) * kEntryWaves + wave;
    const int32_t row = token < tokens ? place[token] : -1;
    const int64_t first = token * teacher.entries;
    if (row >= 0) {
        const TeacherRow r = teacher_row(teacher, token, lane);
        for (int k = lane; k < teacher.entries; k += 64) {
            const int64_t id = teacher.ids[first + k];
            const bool inside = id != teacher.ignore && id >= 0 && id < teacher.vocab;
            ids[wave][k] = inside ? int32_t(id) : -1;
            shares[wave][k] = inside ? r.share(teacher.logit(first + k) * teacher.inverse) : 0.f;
        }
    }
    __syncthreads();
    if (row < 0) return;
    const float base = lse[row], f = factor[row];
    for (int k = lane; k < teacher.entries; k += 64) {
        const int64_t column = int64_t(ids[wave][k]) - from;
        if (column < 0 || column >= columns || ids[wave][k] < 0) continue;
        float q = 0.f;
        bool again = false;
        for (int j = 0; j < teacher.entries; j++) {
            if (ids[wave][j] != ids[wave][k]) continue;
            q += shares[wave][j];
            again |= j < k;
        }
        if (!again) delta[row * piece + column] = T((lifted<T>(picked[first + k] * teacher.inverse, base) - q * float(1 << lift_of<T>)) * f);
    }
}

Teacher teacher_of(const DistillLayout &l, const DistillBuffers &b)
{
    return Teacher{b.ids, b.teacher, l.entries, b.teacher_dt, b.ignore, l.head.vocab, 1.f / b.temperature};
}

hipError_t mark(const DistillLayout &l, const DistillBuffers &b, hipStream_t stream)
{
    mark_tokens<<<dim3(uint32_t((l.head.tokens + 3) / 4)), 256, 0, stream>>>(teacher_of(l, b), l.head.tokens,
                                                                             reinterpret_cast<int64_t *>(b.workspace + l.mark));
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
    const Calls<T, Tempered> calls{l.head, h, stream, Tempered{teacher.inverse}};
    hipError_t error = calls.direct() ? hipSuccess : mark(l, b, stream);
    const int side = calls.loss_parts();
    const int64_t parts = (l.head.vocab + side - 1) / side;
    const auto join = [&](auto waves) {
        constexpr int WAVES = decltype(waves)::value;
        join_divergence<T, WAVES><<<dim3(uint32_t(l.head.tokens)), 64 * WAVES, 0, stream>>>(
            teacher, calls.direct() ? nullptr : calls.template at<int32_t>(l.head.place), parts, l.head.parts, calls.template at<float2>(l.head.stats),
            static_cast<const T *>(b.hidden), static_cast<const T *>(b.weight), l.head.width, loss, lse, picked);
        calls.launched();
    };
    if (calls.direct()) join(std::integral_constant<int, 16>());
    else join(std::integral_constant<int, 4>());
    if (error == hipSuccess) error = calls.error;
    return error;
}

template <typename T>
hipError_t gradient_of(const DistillLayout &l, const DistillBuffers &b, const float *lse, const float *picked, const float *dloss, void *dhidden,
                       void *dweight, hipStream_t stream)
{
    const HeadBuffers h = head_of(l, b);
    const Teacher teacher = teacher_of(l, b);
    const Calls<T, Tempered> calls{l.head, h, stream, Tempered{teacher.inverse}};
    const hipError_t marked = l.head.tokens ? mark(l, b, stream) : hipSuccess;
    const hipError_t rest = calls.gradient(lse, dloss, static_cast<T *>(dhidden), static_cast<T *>(dweight), teacher.inverse, [&](int64_t first, int64_t columns) {
        delta_entries<T><<<dim3(uint32_t((l.head.tokens + kEntryWaves - 1) / kEntryWaves)), 64 * kEntryWaves, 0, stream>>>(
            teacher, calls.template at<int32_t>(l.head.place), l.head.tokens, calls.template at<float>(l.head.lse),
            calls.template at<float>(l.head.factor), picked, first, columns, calls.template at<T>(l.head.delta), l.head.piece);
        calls.launched();
    });
    return marked != hipSuccess ? marked : rest;
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
    if (l.head.dt == CGX_F32) return gradient_of<float>(l, b, lse, picked, dloss, dhidden, dweight, s);
    if (l.head.dt == CGX_F16) return gradient_of<_Float16>(l, b, lse, picked, dloss, dhidden, dweight, s);
    return gradient_of<__bf16>(l, b, lse, picked, dloss, dhidden, dweight, s);
}

}  // namespace cgx
