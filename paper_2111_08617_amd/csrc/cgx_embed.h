// The embedding's calls (include/cgx.h, cgx_embed*): sizes and workspace layout, and launchers (cgx_embed.hip).
#pragma once

#include <cstddef>
#include <cstdint>

#include "../../include/cgx.h"

namespace cgx {

constexpr int kEmbedSortBlocks = 256;                // compute units: each sorts the tokens of its share of the vocabulary
constexpr int kEmbedParts = 256;                     // that many tokens are cut into before they are sorted: a block each
constexpr int64_t kEmbedManyTokens = 24576;          // from which on
constexpr int kEmbedMostChunk = 64;                  // sorted tokens that a wave sums at most: a lane holds each of them

struct SortedToken {
    int32_t id, token;
};

// Sizes of a gradient call and where everything lies in its workspace (offsets in bytes, multiples of 256).
struct EmbedLayout {
    int64_t tokens = 0, width = 0, vocab = 0;
    int dt = 0;
    bool parts = false;      // tokens are first sorted by share, in parts
    int64_t share = 0;       // entries of the vocabulary that a block sorts (a power of two, if there are parts)
    int32_t blocks = 0;      // that sort
    int32_t bits = 0;        // of a place within a share
    int32_t strips = 0;      // of 64 x 16 bytes that a row consists of
    int32_t chunk = 0;       // sorted tokens that a wave sums
    int64_t chunks = 0;
    int64_t pitch = 0;       // floats of a partial row
    size_t list[2] = {0, 0};     // SortedToken [tokens]: tokens, sorted by id; the second is where a sort of several passes goes in between
    size_t part = 0;         // SortedToken [tokens], where there are parts: each part's tokens, sorted by share
    size_t starts = 0;       // uint32 [shares + 1][kEmbedParts]: where a share begins in a part
    size_t partial = 0;      // float [chunks][2][pitch]: sums of the rows that a chunk shares with the one before, and with the one after
    size_t bytes = 0;
};

// CGX_OK and the layout, or the error of the sizes.
int embed_layout(int64_t tokens, int64_t width, int64_t vocab, int dt, EmbedLayout *out);

// The stream is a hipStream_t; the result a hipError_t.
int launch_embed(const void *table, const int64_t *ids, int64_t tokens, int64_t width, int64_t vocab, int dt, int64_t ignore, float scale,
                 void *out, void *stream);
int launch_embed_grad(const EmbedLayout &l, const void *dout, const int64_t *ids, int64_t ignore, float scale, bool accumulate, void *dtable,
                      unsigned char *workspace, void *stream);

}  // namespace cgx
