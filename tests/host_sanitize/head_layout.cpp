// Driver for the sanitizer test of the head's workspace layout: sections in order, without overlap, large enough.
#include <cstdio>
#include <cstdlib>
#include <initializer_list>

#include "../../paper_2111_08617_amd/csrc/cgx_head.h"

static void check(bool ok, const char *what, long long n, long long h, long long v)
{
    if (ok) return;
    std::printf("failed: %s at %lld x %lld x %lld\n", what, n, h, v);
    std::exit(1);
}

int main()
{
    for (int dt : {CGX_F32, CGX_F16, CGX_BF16})
        for (bool grad : {false, true})
            for (long long n : {0ll, 1ll, 63ll, 64ll, 65ll, 255ll, 256ll, 257ll, 4096ll, 100003ll, (1ll << 24) - 1, 1ll << 24, -1ll})
                for (long long h : {0ll, 1ll, 31ll, 32ll, 64ll, 519ll, 2048ll, 1ll << 17, (1ll << 17) + 1})
                    for (long long v : {0ll, 1ll, 255ll, 256ll, 50257ll, 1ll << 20, (1ll << 31) - 257, 1ll << 31}) {
                        cgx::HeadLayout l;
                        if (cgx::head_layout(n, h, v, dt, grad, &l) != CGX_OK) continue;
                        const size_t size = cgx::head_element(dt), rows = size_t(l.rows), pitch = size_t(l.pitch), piece = size_t(l.piece);
                        check(l.rows >= n && l.rows % 256 == 0 && l.pitch >= h && l.pitch % cgx::head_depth(dt) == 0, "rows", n, h, v);
                        check(l.padded == (l.pitch != h) && l.piece % 256 == 0 && l.pieces >= 1, "pieces", n, h, v);
                        check((l.pieces - 1) * l.piece < v && l.pieces * l.piece >= v, "the pieces cover the vocabulary", n, h, v);
                        long long sum = 0;
                        if (l.pieces < 100000)
                            for (long long k = 0; k < l.pieces; k++) sum += l.columns(k);
                        check(l.pieces >= 100000 || sum == v, "columns", n, h, v);
                        check(piece * size * 256 < (size_t(1) << 32) && pitch * size * 256 < (size_t(1) << 32), "offsets of 32 bits", n, h, v);
                        const size_t first[] = {l.place, l.target, l.lse, l.factor, l.picked, l.hidden};
                        const size_t bytes[] = {size_t(n) * 4, rows * 4, rows * 4, rows * 4, rows * 4, rows * pitch * size};
                        size_t end = cgx::kHeadHeaderBytes;
                        for (int k = 0; k < 6; k++) {
                            check(first[k] >= end && first[k] % 256 == 0, "sections", n, h, v);
                            end = first[k] + bytes[k];
                        }
                        if (l.padded) {
                            check(l.weight >= end, "weight", n, h, v);
                            end = l.weight + piece * pitch * size;
                        }
                        check(l.stats >= end && l.stats + size_t(l.parts) * rows * 8 <= l.bytes, "stats", n, h, v);
                        if (!grad) continue;
                        check(l.delta >= end && l.sums >= l.delta + rows * piece * size && l.spare >= l.sums + rows * pitch * 4, "gradient", n, h, v);
                        const size_t split = size_t(cgx::kHeadBlocks) * 256 * 256 * 4;
                        check(l.spare >= l.sums + split && l.spare + split <= l.bytes, "parts", n, h, v);
                    }
    std::printf("all checks passed\n");
    return 0;
}
