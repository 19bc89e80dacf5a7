// Sizes and workspace layout of the calls that learn from a teacher's entries (host only).
#include "cgx_distill.h"

namespace cgx {

int distill_layout(int64_t tokens, int64_t width, int64_t vocab, int32_t entries, int dt, bool grad, DistillLayout *out)
{
    DistillLayout l;
    const int rc = head_layout(tokens, width, vocab, dt, grad, &l.head);
    if (rc != CGX_OK) return rc;
    if (entries < 1 || entries > kMostEntries || tokens * entries >= int64_t(1) << 31) return CGX_ERR_SIZE;
    l.entries = entries;
    l.strips = (vocab + 511) / 512 * 8;
    size_t at = l.head.bytes;
    const auto take = [&at](int64_t bytes) {
        const size_t here = at;
        at += size_t((bytes + 255) / 256 * 256);
        return here;
    };
    l.mark = take(tokens * 8);
    l.token = take(tokens * 4);
    l.entry = take(tokens * entries * 8 + 16);           // (they are read in pairs)
    // the strips are the loss's, what follows the gradient call's; a workspace for that is one for both
    const size_t shared = at;
    l.strip = take(tokens * l.strips * 2);
    size_t end = at;
    if (grad) {
        at = shared;
        l.share = take(tokens * entries * 4);
        l.lower = dt != CGX_F32 && tokens > 0 && tokens <= kLowerTokens;
        l.other = dt == CGX_BF16 && tokens > kLowerTokens;
        if (l.other) {
            l.most = take(2 * kConvertBlocks * 4);
            l.scales = take(2 * 4);
            l.hidden16 = take(l.head.rows * l.head.pitch * 2);
            l.weight16 = take(l.head.piece * l.head.pitch * 2);
        }
        end = at > end ? at : end;
    }
    l.bytes = end;
    *out = l;
    return CGX_OK;
}

}  // namespace cgx
