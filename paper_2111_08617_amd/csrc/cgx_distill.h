// The head's calls that learn from a teacher's entries (include/cgx.h, cgx_head_distill*): sizes and workspace layout, and
// launchers (cgx_distill.hip).
#pragma once

#include "cgx_head.h"

namespace cgx {

constexpr int kMostEntries = 1024;                   // of the teacher, a token

struct DistillLayout {
    HeadLayout head;
    int32_t entries = 0;
    int64_t strips = 0;      // of 64 columns of the vocabulary, rounded up to a multiple of 8
    size_t mark = 0;         // int64 [tokens]: what the head's list reads as targets: kTakesPart, kNoPart or (kWrong) not a number
    size_t token = 0;        // int32 [tokens]: of a row of the list
    size_t entry = 0;        // Entry [tokens][entries]: sorted by id; those that are none are the last, with an id of -1
    size_t share = 0;        // float [tokens][entries] (gradient): of the entries in that order; ids that come again have theirs added to the first
    size_t strip = 0;        // uint16 [tokens][strips] (loss): see Picks
    bool lower = false;      // (gradient) d is held in two parts, see Calls
    bool other = false;      // (gradient) d, and the operands of its products, are held in binary16 instead of bfloat16
    size_t most = 0;         // float [2][kConvertBlocks]: the largest magnitudes that the blocks of a conversion have seen
    size_t scales = 0;       // float [2]: of the converted hidden states and of the weight's piece
    size_t hidden16 = 0;     // binary16 [rows][pitch]
    size_t weight16 = 0;     // binary16 [piece][pitch]
    size_t bytes = 0;
};

// us of the call with gradients with 128, 256, 512 and 1024 blocks, the same inputs again and again: 615 of 4096 x 768 x 30522 228, 230, 233
// and 236 (242 with a launch of its own), 8192 x 2048 x 50257 5495, 5487, 5488 and 5474 (5496).  (With other inputs from pass to pass the calls
// with 256 take 250 and 5640.)
constexpr int kConvertBlocks = 256;
// Up to this many tokens of a gradient are not listed, and hold a 16-bit d in two parts: rows for both are there.  us of loss and gradients (the
// same inputs again and again) with two parts and, for bfloat16 in binary16, for binary16 in one: 128 x 2048 x 50257 326 and 403, 330 and 326;
// 256 x 2048 x 50257 458 and 438, 465 and 340.
constexpr int64_t kLowerTokens = 128;

// CGX_OK and the layout, or the error of the sizes.
int distill_layout(int64_t tokens, int64_t width, int64_t vocab, int32_t entries, int dt, bool grad, DistillLayout *out);

// Device addresses of a call, and its temperature.
struct DistillBuffers {
    const void *hidden, *weight;
    const int64_t *ids;
    const void *teacher;
    int teacher_dt;
    int64_t ignore;
    float temperature;
    unsigned char *workspace;
};
// The stream is a hipStream_t; the result a hipError_t.
int launch_distill(const DistillLayout &l, const DistillBuffers &b, float *loss, float *lse, float *picked, void *stream);
int launch_distill_grad(const DistillLayout &l, const DistillBuffers &b, const float *lse, const float *picked, const float *dloss,
                        void *dhidden, void *dweight, void *stream);

}  // namespace cgx
