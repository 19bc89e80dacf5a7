// Sizes and workspace layout of the head's calls (host only).
#include "cgx_head.h"

namespace cgx {

namespace {

int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// Bytes of d that a call keeps at a time.  A piece is as long as this allows, within [kHeadRows, the vocabulary].
constexpr int64_t kDeltaBytes = int64_t(512) << 20;

}  // namespace

int head_layout(int64_t tokens, int64_t width, int64_t vocab, int dt, bool grad, HeadLayout *out)
{
    if (dt != CGX_F32 && dt != CGX_F16 && dt != CGX_BF16) return CGX_ERR_DTYPE;
    if (tokens < 0 || tokens >= (int64_t(1) << 24) || width < 1 || width > (1 << 17) || vocab < 1 || vocab >= int64_t(1) << 28)
        return CGX_ERR_SIZE;
    const int64_t size = int64_t(head_element(dt));
    HeadLayout l;
    l.tokens = tokens;
    l.width = width;
    l.vocab = vocab;
    l.dt = dt;
    l.rows = up(tokens > 0 ? tokens : 1, kHeadRows);
    l.pitch = up(width, head_depth(dt));
    l.padded = l.pitch != width;
    // a launch has a block of 256 threads per 64 x 64 results, begun ones among them, at most, and fewer than 2^32 threads
    if (l.rows * up(vocab, 64) >= int64_t(1) << 36 || l.rows * up(width, 64) >= int64_t(1) << 36) return CGX_ERR_SIZE;
    // pieces of about the same length; at most 2^18 columns, so that byte offsets within a tile's rows fit 32 bits
    int64_t most = kDeltaBytes / (l.rows * size) / kHeadRows * kHeadRows;
    most = most < kHeadRows ? kHeadRows : most > (1 << 18) ? (1 << 18) : most;
    l.pieces = (vocab + most - 1) / most;
    l.piece = up((vocab + l.pieces - 1) / l.pieces, kHeadRows);
    l.pieces = (vocab + l.piece - 1) / l.piece;
    // columns of the narrowest tile, or of a block of the kernel for few tokens
    const int64_t narrowest = tokens <= kDirectTokens || ((tokens + 63) / 64) * ((vocab + 63) / 64) <= kFewTiles ? kFewColumns : 64;
    l.parts = (vocab + narrowest - 1) / narrowest;
    size_t at = kHeadHeaderBytes;
    const auto take = [&at](int64_t bytes) {
        const size_t here = at;
        at += size_t(up(bytes, 256));
        return here;
    };
    l.place = take(tokens * 4);
    l.target = take(l.rows * 4);
    l.lse = take(l.rows * 4);
    l.factor = take(l.rows * 4);
    l.picked = take(l.rows * 4);
    l.hidden = take(l.rows * l.pitch * size);
    l.weight = l.padded ? take(l.piece * l.pitch * size) : 0;
    // the forward call's partial sums and the gradient call's pieces are never needed together
    const size_t shared = at;
    l.stats = take(l.parts * l.rows * 8);
    size_t end = at;
    if (grad) {
        at = shared;
        l.delta = take(l.rows * l.piece * size);
        // (whole tiles of the blocks that a split sum fills, or all rows)
        const int64_t split = int64_t(kHeadBlocks) * kHeadRows * kHeadRows, rows = l.rows * l.pitch;
        l.sums = take((split > rows ? split : rows) * 4);
        l.spare = take(split * 4);
        end = at > end ? at : end;
    }
    l.bytes = end;
    *out = l;
    return CGX_OK;
}

}  // namespace cgx
