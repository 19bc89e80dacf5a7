// Sizes and workspace layout of the calls that learn from a teacher's entries (host only).
#include "cgx_distill.h"

namespace cgx {

int distill_layout(int64_t tokens, int64_t width, int64_t vocab, int32_t entries, int dt, bool grad, DistillLayout *out)
{
    DistillLayout l;
    const int rc = head_layout(tokens, width, vocab, dt, grad, &l.head);
    if (rc != CGX_OK) return rc;
    if (entries < 1 || entries > kMostEntries) return CGX_ERR_SIZE;
    l.entries = entries;
    l.mark = l.head.bytes;
    l.bytes = l.mark + size_t((tokens * 8 + 255) / 256 * 256);
    *out = l;
    return CGX_OK;
}

}  // namespace cgx
