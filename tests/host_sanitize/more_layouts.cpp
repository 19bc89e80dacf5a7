// Workspaces of the embedding's gradient and of distillation: on many sizes, sections lie one behind another, aligned, within the bytes reported, and are
// as long as what the kernels write there.
#include <cstdio>
#include <cstdlib>
#include <algorithm>
#include <random>
#include <utility>
#include <vector>

#include "../../paper_2111_08617_amd/csrc/cgx_distill.h"
#include "../../paper_2111_08617_amd/csrc/cgx_embed.h"

using namespace cgx;

#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s failed\n", __LINE__, #x); std::exit(1); } } while (0)

using Sections = std::vector<std::pair<size_t, int64_t>>;       // offset, bytes

static void disjoint(Sections s, size_t bytes, size_t from)
{
    std::sort(s.begin(), s.end());
    size_t at = from;
    for (const auto &[offset, length] : s) {
        CHECK(length >= 0 && offset % 256 == 0 && offset >= at);
        at = offset + size_t(length);
    }
    CHECK(at <= bytes);
}

static int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

static bool embed(int64_t n, int64_t h, int64_t v, int dt)
{
    EmbedLayout l;
    const bool fits = n >= 0 && n < 1 << 24 && h >= 1 && h <= 1 << 17 && v >= 1 && v < 1 << 28 && n * h < int64_t(1) << 35 && v * h < int64_t(1) << 35;
    const int rc = embed_layout(n, h, v, dt, &l);
    CHECK(rc == (fits ? CGX_OK : CGX_ERR_SIZE));
    if (!fits) return false;
    CHECK(l.blocks >= 1 && l.blocks <= kEmbedSortBlocks && int64_t(l.blocks) * l.share >= v && int64_t(l.blocks - 1) * l.share < v);
    CHECK((int64_t(1) << l.bits) >= l.share && (l.bits == 0 || (int64_t(1) << (l.bits - 1)) < l.share));
    CHECK(l.chunk >= 8 && l.chunk <= kEmbedMostChunk && l.chunk % 8 == 0 && l.chunks * l.chunk >= n && (l.chunks - 1) * l.chunk < std::max<int64_t>(n, 1));
    CHECK(l.pitch >= h && l.strips * (dt == CGX_F32 ? 256 : 512) == l.pitch);
    // launches: fewer than 2^32 threads each
    const int64_t fills = (v * h * (dt == CGX_F32 ? 4 : 2) + 65535) / 65536;
    CHECK((fills + l.blocks) * 1024 < int64_t(1) << 32 && l.chunks * l.strips * 512 < int64_t(1) << 32 && (l.chunks * l.strips + 4) * 64 < int64_t(1) << 32);
    Sections s{{l.list[0], n * 8}, {l.partial, l.chunks * 2 * l.pitch * 4}};
    if (l.bits > 8) s.push_back({l.list[1], n * 8});
    CHECK(l.parts == (n > kEmbedManyTokens));
    if (l.parts) {
        CHECK((l.share & (l.share - 1)) == 0 && l.share == int64_t(1) << l.bits && ((v - 1) >> l.bits) < 256);
        s.push_back({l.part, n * 8});
        s.push_back({l.starts, (l.blocks + 1) * int64_t(kEmbedParts) * 4});
    }
    disjoint(s, l.bytes, 256);
    return true;
}

static bool distill(int64_t n, int64_t h, int64_t v, int32_t k, int dt, bool grad)
{
    DistillLayout l;
    HeadLayout head;
    const int of_head = head_layout(n, h, v, dt, grad, &head);
    const bool fits = of_head == CGX_OK && k >= 1 && k <= kMostEntries && n * k < int64_t(1) << 31;
    const int rc = distill_layout(n, h, v, k, dt, grad, &l);
    CHECK(rc == (fits ? CGX_OK : CGX_ERR_SIZE));
    if (!fits) return false;
    CHECK(l.head.bytes == head.bytes && l.entries == k && l.strips % 8 == 0 && l.strips * 64 >= v);
    Sections s{{l.mark, n * 8}, {l.token, n * 4}, {l.entry, n * k * 8 + 16}};
    if (!grad) s.push_back({l.strip, n * l.strips * 2});
    if (grad) s.push_back({l.share, n * k * 4});
    if (l.lower) {
        // two parts of d, and the hidden states twice, in the rows that are there
        const int64_t lower = up(n, 64);
        CHECK(grad && dt != CGX_F32 && n > 0 && 2 * lower <= l.head.rows);
    }
    CHECK(l.other == (grad && dt == CGX_BF16 && n > kLowerTokens));
    if (l.other) {
        s.push_back({l.most, 2 * kConvertBlocks * 4});
        s.push_back({l.scales, 8});
        s.push_back({l.hidden16, l.head.rows * l.head.pitch * 2});
        s.push_back({l.weight16, l.head.piece * l.head.pitch * 2});
    }
    disjoint(s, l.bytes, l.head.bytes);
    DistillLayout loss;
    CHECK(distill_layout(n, h, v, k, dt, false, &loss) == CGX_OK && loss.bytes <= l.bytes);      // (for both calls)
    return true;
}

int main()
{
    std::mt19937_64 g(11);
    const auto any = [&](int64_t lo, int64_t hi) {              // spread over the logarithm
        const double u = double(g() >> 11) * 0x1p-53;
        int64_t v = lo;
        while (v < hi && double(g() >> 11) * 0x1p-53 < 0.93 - 0.2 * u) v = v < 8 ? v + 1 : v + v / 4 + int64_t(g() % 3);
        return std::min(v, hi);
    };
    int taken = 0, refused = 0;
    for (int i = 0; i < 60000; i++) {
        const int64_t n = any(0, (1 << 24) + 3), h = any(1, (1 << 17) + 3), v = any(1, (1 << 28) + 3);
        const int dt = int(g() % 3);
        (embed(n, h, v, dt) ? taken : refused)++;
        (distill(n, h, v, int32_t(any(0, 1027)), dt, g() % 2) ? taken : refused)++;
    }
    for (int64_t n : {0, 1, 8, 63, 64, 65, 128, 129, 255, 16384, 16385, (1 << 24) - 1})
        for (int64_t v : {1, 2, 255, 256, 257, 65536, 65537, (1 << 24) + 1, (1 << 28) - 1})
            for (int64_t h : {1, 127, 128, 2048})
                for (int dt : {0, 1, 2}) {
                    embed(n, h, v, dt);
                    for (int k : {1, 64, 65, 1024}) distill(n, h, v, k, dt, true), distill(n, h, v, k, dt, false);
                }
    std::printf("all checks passed, %d taken %d refused\n", taken, refused);
}
