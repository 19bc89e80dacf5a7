// The head's calls (include/cgx.h, cgx_head_*): sizes and workspace layout (host only, cgx_head.cpp) and launchers (cgx_head.hip).
#pragma once

#include <cstddef>
#include <cstdint>

#include "../../include/cgx.h"

namespace cgx {

constexpr int kHeadRows = 256;                       // token rows and columns of a piece come in multiples of it (the largest tile)
constexpr int kHeadBlocks = 256;                     // compute units: a sum is split into parts where its tiles are fewer
constexpr size_t kHeadHeaderBytes = 256;
constexpr int kDirectTokens = 64;                    // up to this many tokens the loss can take as they come
constexpr int kFewTokens = 16;                       // a block of its kernel for few tokens takes this many, and
constexpr int kFewColumns = 32;                      // this many columns of the vocabulary
constexpr int kFewTiles = 64;                        // it also takes calls of up to this many tiles of 64 x 64 logits

inline size_t head_element(int dt) { return dt == CGX_F32 ? 4 : 2; }
// Elements of the summed axis per step of the products: rows are padded to a multiple of it.
inline int64_t head_depth(int dt) { return int64_t(128 / head_element(dt)); }

// Sizes of a call and where everything lies in its workspace (offsets in bytes, multiples of 256).
struct HeadLayout {
    int64_t tokens = 0, width = 0, vocab = 0;
    int dt = 0;
    int64_t rows = 0;        // tokens, rounded up to whole tiles
    int64_t pitch = 0;       // elements of a padded row of hidden states or weights
    bool padded = false;     // the weight has to be copied into padded rows, piece by piece
    int64_t piece = 0;       // columns of a piece of the vocabulary (a multiple of kHeadRows)
    int64_t pieces = 0;
    int64_t parts = 0;       // partial sums per token of the forward call
    size_t place = 0;        // int32 [tokens]: row of a token, or -1; rows are the tokens that count, in order
    size_t target = 0;       // int32 [rows]: -1 where the target is outside the vocabulary
    size_t lse = 0;          // float [rows]
    size_t factor = 0;       // float [rows]: dloss in the units of d
    size_t picked = 0;       // float [rows]: the target's logit
    size_t hidden = 0;       // T [rows][pitch]
    size_t weight = 0;       // T [piece][pitch], where padded
    size_t stats = 0;        // float2 [rows][parts]: largest logit of a part, and the sum of exp(logit - it)
    size_t delta = 0;        // T [rows][piece]: d of a piece
    size_t sums = 0;         // float [parts][rows][pitch]: dhidden while it is summed, in parts of the vocabulary if tokens are few
    size_t spare = 0;        // float [blocks][tile]: parts of tiles of the weight's gradient
    size_t bytes = 0;
    int64_t columns(int64_t k) const { return k + 1 < pieces ? piece : vocab - (pieces - 1) * piece; }
};

// CGX_OK and the layout, or the error of the sizes.
int head_layout(int64_t tokens, int64_t width, int64_t vocab, int dt, bool grad, HeadLayout *out);

// Device addresses of a call.
struct HeadBuffers {
    const void *hidden, *weight;
    const int64_t *targets;
    int64_t ignore;
    unsigned char *workspace;
};
// The stream is a hipStream_t; the result a hipError_t.
int launch_head_loss(const HeadLayout &l, const HeadBuffers &b, float *loss, float *lse, void *stream);
int launch_head_loss_grad(const HeadLayout &l, const HeadBuffers &b, const float *lse, const float *dloss, void *dhidden,
                          void *dweight, void *stream);

}  // namespace cgx
