// extern "C" entry points of what stands beside the fused buffer (see include/cgx.h): the head's loss and its gradient,
// the gradients' norm and clipping.  Argument checks, then launches on the caller's stream.
#include <hip/hip_runtime.h>

#include "cgx_grad.h"
#include "cgx_head.h"

namespace {

bool misaligned(const void *p, uintptr_t to = 16) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

int status_of(int e) { return e == hipSuccess ? CGX_OK : CGX_ERR_HIP; }

bool known_type(int dt) { return dt == CGX_F32 || dt == CGX_F16 || dt == CGX_BF16; }

// A list of tensors: the calls read and write nothing before all of it has been checked.
int check_tensors(const cgx_tensor *tensors, int32_t count)
{
    if (count < 0) return CGX_ERR_SIZE;
    if (count > 0 && !tensors) return CGX_ERR_NULL;
    for (int32_t k = 0; k < count; k++) {
        const cgx_tensor &t = tensors[k];
        if (!known_type(t.dt)) return CGX_ERR_DTYPE;
        if (t.n < 0 || t.n >= (int64_t(1) << 43)) return CGX_ERR_SIZE;
        if (t.n > 0 && !t.data) return CGX_ERR_NULL;
        if (t.n > 0 && misaligned(t.data, t.dt == CGX_F32 ? 4 : 2)) return CGX_ERR_ALIGN;
    }
    return CGX_OK;
}

}  // namespace

extern "C" {

int cgx_head_workspace(int64_t tokens, int32_t width, int64_t vocab, cgx_dtype dt, int32_t grad, size_t *bytes)
{
    cgx::HeadLayout l;
    const int rc = cgx::head_layout(tokens, width, vocab, int(dt), grad != 0, &l);
    if (rc != CGX_OK) return rc;
    if (!bytes) return CGX_ERR_NULL;
    *bytes = l.bytes;
    return CGX_OK;
}

int cgx_head_loss(const void *hidden, const void *weight, const int64_t *targets, int64_t tokens, int32_t width, int64_t vocab,
                  cgx_dtype dt, int64_t ignore, float *loss, float *lse, void *workspace, size_t workspace_bytes, void *stream)
{
    cgx::HeadLayout l;
    const int rc = cgx::head_layout(tokens, width, vocab, int(dt), false, &l);
    if (rc != CGX_OK) return rc;
    if (tokens == 0) return CGX_OK;
    if (!hidden || !weight || !targets || !loss || !lse || !workspace) return CGX_ERR_NULL;
    if (misaligned(hidden) || misaligned(weight) || misaligned(workspace) || misaligned(targets, 8) || misaligned(loss, 4) ||
        misaligned(lse, 4))
        return CGX_ERR_ALIGN;
    if (workspace_bytes < l.bytes) return CGX_ERR_SIZE;
    return status_of(cgx::launch_head_loss(l, {hidden, weight, targets, ignore, static_cast<unsigned char *>(workspace)}, loss, lse, stream));
}

int cgx_head_loss_grad(const void *hidden, const void *weight, const int64_t *targets, const float *lse, const float *dloss,
                       int64_t tokens, int32_t width, int64_t vocab, cgx_dtype dt, int64_t ignore, void *dhidden, void *dweight,
                       void *workspace, size_t workspace_bytes, void *stream)
{
    cgx::HeadLayout l;
    const int rc = cgx::head_layout(tokens, width, vocab, int(dt), true, &l);
    if (rc != CGX_OK) return rc;
    if (!weight || !dweight || !workspace) return CGX_ERR_NULL;
    if (tokens > 0 && (!hidden || !targets || !lse || !dloss || !dhidden)) return CGX_ERR_NULL;
    if (misaligned(hidden) || misaligned(weight) || misaligned(workspace) || misaligned(dhidden) || misaligned(dweight) ||
        misaligned(targets, 8) || misaligned(lse, 4) || misaligned(dloss, 4))
        return CGX_ERR_ALIGN;
    if (workspace_bytes < l.bytes) return CGX_ERR_SIZE;
    return status_of(cgx::launch_head_loss_grad(l, {hidden, weight, targets, ignore, static_cast<unsigned char *>(workspace)}, lse, dloss,
                                                dhidden, dweight, stream));
}

int cgx_grad_norm_workspace(size_t *bytes)
{
    if (!bytes) return CGX_ERR_NULL;
    *bytes = size_t(cgx::kNormSlots) * sizeof(double);
    return CGX_OK;
}

int cgx_grad_norm(const cgx_tensor *tensors, int32_t count, float *norm, void *workspace, size_t workspace_bytes, void *stream)
{
    const int rc = check_tensors(tensors, count);
    if (rc != CGX_OK) return rc;
    if (!norm || !workspace) return CGX_ERR_NULL;
    if (misaligned(norm, 4) || misaligned(workspace)) return CGX_ERR_ALIGN;
    if (workspace_bytes < size_t(cgx::kNormSlots) * sizeof(double)) return CGX_ERR_SIZE;
    return status_of(cgx::launch_grad_norm(tensors, count, norm, static_cast<double *>(workspace), static_cast<hipStream_t>(stream)));
}

int cgx_grad_clip(const cgx_tensor *tensors, int32_t count, const float *norm, float max_norm, void *out, cgx_dtype out_dt,
                  void *stream)
{
    const int rc = check_tensors(tensors, count);
    if (rc != CGX_OK) return rc;
    if (!(max_norm >= 0.f)) return CGX_ERR_SIZE;
    if (out && !known_type(int(out_dt))) return CGX_ERR_DTYPE;
    if (!norm) return CGX_ERR_NULL;
    if (misaligned(norm, 4) || misaligned(out)) return CGX_ERR_ALIGN;
    return status_of(cgx::launch_grad_clip(tensors, count, norm, max_norm, out, int(out_dt), static_cast<hipStream_t>(stream)));
}

}  // extern "C"
