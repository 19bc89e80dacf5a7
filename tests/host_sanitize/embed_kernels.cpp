// The embedding's kernels, lane by lane on the CPU: lists, parts, starts, partial rows, tables and outputs are allocations of
// exactly the size that the layout gives them, so that the sanitizers see every access outside.
#include "embed_kernels.inc"                             // cgx_embed.hip without its launches

using namespace cgx;

namespace {

#define CHECK(x) do { if (!(x)) { std::printf("failed: %s (line %d)\n", #x, __LINE__); std::abort(); } } while (0)

template <class T>
struct Exactly {                                         // n elements and not one more; garbage to begin with
    T *p;
    explicit Exactly(size_t n) : p(static_cast<T *>(std::malloc(n * sizeof(T) ? n * sizeof(T) : 1)))
    {
        std::memset(static_cast<void *>(p), 0xa5, n * sizeof(T));
    }
    ~Exactly() { std::free(p); }
    Exactly(const Exactly &) = delete;
    operator T *() const { return p; }
};

struct Call {
    int64_t tokens, width, vocab, ignore;
    bool accumulate;
};

// As launch_embed_grad does it; `sorted` says whether few tokens are to be sorted as well.
void gradient(const Call &c, const std::vector<int64_t> &given, std::mt19937_64 &g, bool sorted)
{
    EmbedLayout l;
    CHECK(embed_layout(c.tokens, c.width, c.vocab, CGX_F32, &l) == CGX_OK);
    const size_t n = size_t(c.tokens), h = size_t(c.width), v = size_t(c.vocab);
    Exactly<int64_t> ids(n);
    Exactly<float> dout(n * h), dtable(v * h);
    std::copy(given.begin(), given.end(), ids.p);
    const auto there = [&](int64_t id) { return id >= 0 && id < c.vocab && id != c.ignore; };
    for (size_t k = 0; k < n; k++)
        for (size_t e = 0; e < h; e++) dout[k * h + e] = there(ids[k]) ? float(int(g() % 17) - 8) : __builtin_nanf("");
    std::vector<float> want(v * h);
    for (size_t k = 0; k < v * h; k++) dtable[k] = want[k] = c.accumulate ? float(int(g() % 9) - 4) : __builtin_nanf("");
    if (!c.accumulate) std::fill(want.begin(), want.end(), 0.f);
    for (size_t k = 0; k < n; k++)                       // (whole numbers: exact in any order)
        if (there(ids[k]))
            for (size_t e = 0; e < h; e++) want[size_t(ids[k]) * h + e] += 2.f * dout[k * h + e];
    const bool few = !sorted && c.tokens <= kFewTokens;
    if (few) {
        const int64_t each = c.vocab % 3 ? 1 : 4, items = (c.accumulate ? c.tokens : (c.vocab + each - 1) / each) * l.strips;
        waves::launch(uint32_t((items + 3) / 4), kBlock, &g, [&] {
            few_rows<float>(ids, dout, int32_t(c.tokens), c.ignore, c.vocab, c.width, uint32_t(l.strips), 2.f, c.accumulate,
                            dtable, int32_t(each));
        });
    } else {
        Exactly<EmbedHeader> header(1);
        Exactly<SortedToken> list(n), between(l.list[1] ? n : 0), part(l.parts ? n : 0);
        Exactly<uint32_t> starts(l.parts ? size_t(l.blocks + 1) * kEmbedParts : 0);
        Exactly<float> partial(size_t(l.chunks * 2 * l.pitch));
        const Parts parts{part, starts, uint32_t((l.tokens + kEmbedParts - 1) / kEmbedParts), l.bits};
        const int64_t bytes = c.vocab * c.width * 4, fills = c.accumulate ? 0 : (bytes + kFillBytes - 1) / kFillBytes;
        const uint32_t sorts = uint32_t(l.blocks);
        if (l.parts)
            waves::launch(kEmbedParts, kSortThreads, &g, [&] { sort_parts(ids, uint32_t(n), c.ignore, c.vocab, l.blocks, parts); });
        waves::launch(sorts + uint32_t(fills), kSortThreads, &g, [&] {
            auto *const table = reinterpret_cast<unsigned char *>(dtable.p);
            const auto go = [&](auto fill, auto in_parts) {
                sort_tokens<decltype(fill)::value, decltype(in_parts)::value>(
                    ids, uint32_t(n), c.ignore, c.vocab, l.share, l.bits, sorts, header, list, between, parts, table, bytes);
            };
            const std::true_type yes;
            const std::false_type no;
            if (l.parts) fills ? go(yes, yes) : go(no, yes);
            else fills ? go(yes, no) : go(no, no);
        });
        std::vector<std::pair<int64_t, int32_t>> order;
        for (size_t k = 0; k < n; k++)
            if (there(ids[k])) order.push_back({ids[k], int32_t(k)});
        std::stable_sort(order.begin(), order.end(), [](auto &a, auto &b) { return a.first < b.first; });
        CHECK(header.p->count == int32_t(order.size()));
        for (size_t k = 0; k < order.size(); k++) CHECK(list[k].id == order[k].first && list[k].token == order[k].second);
        const int64_t items = l.chunks * l.strips;
        waves::launch(uint32_t((items + 3) / 4), kBlock, &g, [&] {
            sum_chunks<float>(header, list, dout, c.width, uint32_t(l.strips), l.chunk, 2.f, c.accumulate, dtable, partial,
                              l.pitch);
        });
        if (l.chunks > 1)
            waves::launch(uint32_t((l.chunks - 1) * l.strips), 64 * kJoinWaves, &g, [&] {
                join_runs<float>(header, list, c.width, uint32_t(l.strips), l.chunk, 2.f, c.accumulate, dtable, partial,
                                 l.pitch);
            });
    }
    for (size_t k = 0; k < v * h; k++) CHECK(dtable[k] == want[k]);
}

template <int EACH>
void look_up_some(const Call &c, const std::vector<int64_t> &given, std::mt19937_64 &g)
{
    const size_t n = size_t(c.tokens), h = size_t(c.width), v = size_t(c.vocab);
    Exactly<int64_t> ids(n);
    Exactly<float> table(v * h), out(n * h);
    std::copy(given.begin(), given.end(), ids.p);
    for (size_t k = 0; k < v * h; k++) table[k] = float(g() % 1000);
    const int64_t strips = (c.width + 255) / 256, parts = (strips + EACH - 1) / EACH;
    waves::launch(uint32_t((c.tokens * parts + 3) / 4), kBlock, &g, [&] {
        look_up<float, EACH>(table, ids, c.tokens, c.width, c.vocab, c.ignore, 2.f, uint32_t(parts), out);
    });
    for (size_t k = 0; k < n; k++)
        for (size_t e = 0; e < h; e++) {
            const float got = out[k * h + e];
            if (ids[k] == c.ignore) CHECK(got == 0.f);
            else if (ids[k] < 0 || ids[k] >= c.vocab) CHECK(got != got);
            else CHECK(got == 2.f * table[size_t(ids[k]) * h + e]);
        }
}

std::vector<int64_t> tokens_of(const Call &c, int kind, std::mt19937_64 &g)
{
    std::vector<int64_t> ids(size_t(c.tokens));
    const auto uniform = [&] { return double(g() >> 11) * 0x1p-53; };
    for (auto &id : ids) {
        const double u = uniform(), v = double(c.vocab);
        id = kind == 1 ? c.vocab / 2 : int64_t(kind == 0 ? u * u * u * v : kind == 2 ? u * std::min(v, 3.) : u * v);
        id = std::min(id, c.vocab - 1);
        const uint64_t r = kind == 1 ? 4 : g() % 40;
        if (r == 0) id = c.ignore;
        if (r == 1) id = c.vocab + int64_t(g() % 3);
        if (r == 2) id = -int64_t(g() % 5) - 1;
        if (r == 3) id = (int64_t(1) << 32) + int64_t(g() % uint64_t(c.vocab));
    }
    return ids;
}

}  // namespace

int main()
{
    std::mt19937_64 g(7);
    // sorts by all tokens, of one to three digits, whose shares may be empty; few tokens; rows of one and several strips
    const Call calls[] = {{1, 1, 1, -100, false}, {1, 5, 3, -100, true}, {2, 3, 5, 1, false}, {64, 64, 64, -100, false},
                          {65, 300, 20, 7, true}, {127, 1, 257, -100, false}, {129, 3, 300, -100, false},
                          {300, 260, 40, 5, true}, {700, 2, 30, -100, false}, {1025, 7, 3, -100, true},
                          {3000, 1, 66000, -100, true}, {150, 1, 70000, -100, false}};
    for (const Call &c : calls)
        for (int kind = 0; kind < 4; kind += c.vocab > 64 ? 3 : 1) {
            const std::vector<int64_t> ids = tokens_of(c, kind, g);
            gradient(c, ids, g, true);
            if (c.tokens <= 128) gradient(c, ids, g, false);
            if (c.vocab < 1000) {
                look_up_some<1>(c, ids, g);
                look_up_some<2>(c, ids, g);
                look_up_some<4>(c, ids, g);
            }
        }
    const Call longest = {200, 1, 17000001, -100, true};
    gradient(longest, tokens_of(longest, 3, g), g, true);
    std::printf("sorts by all tokens\n");
    // sorts in parts: short and long shares, parts that end early, one to three digits
    const Call many[] = {{24577, 1, 3, -100, false}, {24700, 2, 259, 4, false}, {25003, 1, 70000, -100, true},
                         {24999, 1, 17000001, -100, true}};
    for (const Call &c : many) gradient(c, tokens_of(c, 0, g), g, true);
    gradient(many[0], tokens_of(many[0], 1, g), g, true);
    std::printf("all checks passed\n");
    return 0;
}
