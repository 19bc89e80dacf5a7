// Sizes and workspace layout of the embedding's calls (host only).
#include "cgx_embed.h"

namespace cgx {

int embed_layout(int64_t tokens, int64_t width, int64_t vocab, int dt, EmbedLayout *out)
{
    if (dt != CGX_F32 && dt != CGX_F16 && dt != CGX_BF16) return CGX_ERR_DTYPE;
    if (tokens < 0 || tokens >= int64_t(1) << 24 || width < 1 || width > 1 << 17 || vocab < 1 || vocab >= int64_t(1) << 28) return CGX_ERR_SIZE;
    // (a launch that writes zeros has a block of 1024 threads per 64 KB, and fewer than 2^32 threads)
    if (vocab * width >= int64_t(1) << 35 || tokens * width >= int64_t(1) << 35) return CGX_ERR_SIZE;
    EmbedLayout l;
    l.tokens = tokens;
    l.width = width;
    l.vocab = vocab;
    l.dt = dt;
    l.share = (vocab + kEmbedSortBlocks - 1) / kEmbedSortBlocks;
    l.parts = tokens > kEmbedManyTokens;
    if (l.parts) {
        int64_t share = 1;
        while (share < l.share) share *= 2;
        l.share = share;
    }
    l.blocks = int32_t((vocab + l.share - 1) / l.share);
    while (int64_t(1) << l.bits < l.share) l.bits++;
    const int64_t columns = dt == CGX_F32 ? 256 : 512;
    l.strips = int32_t((width + columns - 1) / columns);
    // Chunks as long as leaves some thousand waves.  With 2048 and 4096 of them sums and joins of 8192 x 2048 bfloat16 take 12.7 + 5.1 and 11.5 + 7.2 us, of
    // 65536 x 1024 23.4 + 8.0 and 22.8 + 11.6.
    l.chunk = 8;
    while (l.chunk < kEmbedMostChunk && tokens / (2 * l.chunk) * l.strips >= 2048) l.chunk *= 2;
    l.chunks = (tokens + l.chunk - 1) / l.chunk;
    l.pitch = l.strips * columns;
    size_t at = 256;
    const auto take = [&at](int64_t bytes) {
        const size_t here = at;
        at += size_t((bytes + 255) / 256 * 256);
        return here;
    };
    const int arrays = l.bits > 8 ? 2 : 1;
    for (int k = 0; k < arrays; k++) l.list[k] = take(tokens * int64_t(sizeof(SortedToken)));
    if (l.parts) {
        l.part = take(tokens * int64_t(sizeof(SortedToken)));
        l.starts = take((l.blocks + 1) * kEmbedParts * 4);
    }
    l.partial = take(l.chunks * 2 * l.pitch * 4);
    l.bytes = at;
    *out = l;
    return CGX_OK;
}

}  // namespace cgx
