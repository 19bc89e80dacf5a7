// The head's calls with one target a token: softmax cross entropy and its gradient (kernels in cgx_head_kernels.h).
#include "cgx_head_kernels.h"

namespace cgx {

namespace {

template <typename T>
hipError_t gradient_of(const HeadLayout &l, const HeadBuffers &b, const float *lse, const float *dloss, void *dhidden, void *dweight,
                       hipStream_t stream)
{
    const Calls<T> calls{l, b, stream};
    return calls.gradient(static_cast<T *>(dhidden), static_cast<T *>(dweight), [&] { calls.list(dloss, lse); }, [](int64_t, int64_t) { return Nothing(); },
                          [](const T *, int64_t, int64_t) {});
}

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
    if (l.dt == CGX_F32) return gradient_of<float>(l, b, lse, dloss, dhidden, dweight, s);
    if (l.dt == CGX_F16) return gradient_of<_Float16>(l, b, lse, dloss, dhidden, dweight, s);
    return gradient_of<__bf16>(l, b, lse, dloss, dhidden, dweight, s);
}

}  // namespace cgx
