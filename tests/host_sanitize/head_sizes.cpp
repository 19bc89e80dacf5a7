// Driver for the test of the head's limits: which sizes head_layout takes, against limits that are worked out here, and that every launch
// of an accepted size stays under 2^32 threads.  Prints how many sizes were taken and refused.
#include <cstdio>
#include <cstdlib>
#include <initializer_list>

#include "../../paper_2111_08617_amd/csrc/cgx_head.h"

typedef long long ll;
typedef unsigned __int128 wide;          // (no product below can overflow)

static wide up(wide v, wide to) { return (v + to - 1) / to; }

static void check(bool ok, const char *what, ll n, ll h, ll v, int dt)
{
    if (ok) return;
    std::printf("failed: %s at %lld x %lld x %lld, type %d\n", what, n, h, v, dt);
    std::exit(1);
}

// include/cgx.h: tokens < 2^24, 1 <= width <= 2^17, and the tokens, rounded up to a multiple of 256 (one at least), times the vocabulary
// or times the width, both rounded up to a multiple of 64, below 2^36.
static bool allowed(ll n, ll h, ll v)
{
    if (n < 0 || n >= (1ll << 24) || h < 1 || h > (1ll << 17) || v < 1) return false;
    const wide rows = n ? up(wide(n), 256) * 256 : 256, limit = wide(1) << 36;
    return rows * (up(wide(v), 64) * 64) < limit && rows * (up(wide(h), 64) * 64) < limit;
}

static ll accepted, refused;

static void size(ll n, ll h, ll v, int dt)
{
    for (bool grad : {false, true}) {
        cgx::HeadLayout l;
        const int status = cgx::head_layout(n, h, v, dt, grad, &l);
        check(status == (allowed(n, h, v) ? CGX_OK : CGX_ERR_SIZE), "status", n, h, v, dt);
        (status == CGX_OK ? accepted : refused)++;
        if (status != CGX_OK) continue;
        // threads of the launches whose grids grow with the call: 64 x 64 results by 256 threads at most, a token by 256
        const wide limit = wide(1) << 32, tokens = up(wide(n), 64);
        check(tokens * up(wide(v), 64) * 256 < limit, "threads of the logits", n, h, v, dt);
        check(tokens * up(wide(l.piece), 64) * 256 < limit, "threads of a piece", n, h, v, dt);
        check(tokens * up(wide(l.pitch), 64) * 256 < limit, "threads of the hidden states' gradient", n, h, v, dt);
        check((up(wide(l.piece), 64) * up(wide(h), 64) + 1024) * 256 < limit, "threads of the weight's gradient", n, h, v, dt);
        check(wide(n) * 256 < limit && wide(l.piece) * 256 < limit, "threads of rows", n, h, v, dt);
        check(l.pieces >= 1 && wide(l.pieces) * wide(l.piece) >= wide(v), "the pieces cover the vocabulary", n, h, v, dt);
    }
}

int main()
{
    const ll k = 1;
    for (int dt : {CGX_F32, CGX_F16, CGX_BF16}) {
        for (ll n : {-k, 0 * k, k, 63 * k, 64 * k, 65 * k, 200 * k, 256 * k, 257 * k, 8192 * k, 65536 * k, 100003 * k, (k << 24) - 256, (k << 24) - 255, (k << 24) - 1, k << 24, k << 62})
            for (ll h : {-k, 0 * k, k, 31 * k, 32 * k, 64 * k, 519 * k, 2048 * k, 4000 * k, 4032 * k, 4064 * k, k << 17, (k << 17) + 1, k << 62})
                for (ll v : {-k, 0 * k, k, 63 * k, 64 * k, 4032 * k, 4033 * k, 50257 * k, (k << 20) - 64, (k << 20) - 63, (k << 20) - 1, k << 20, (k << 23) - 64, (k << 23) - 1,
                             (k << 28) - 64, (k << 28) - 63, (k << 28) - 1, k << 28, (k << 31) - 257, k << 31, (k << 62) + 5})
                    size(n, h, v, dt);
        // the longest vocabulary and the one after it, for tokens of every length
        for (ll n = 1; n < (k << 24); n = n * 3 + 1) {
            const ll rows = (n + 255) / 256 * 256, most = ((k << 36) - 1) / rows / 64 * 64;
            for (ll v : {most - 1, most, most + 1}) size(n, 96, v, dt);
        }
    }
    std::printf("all checks passed, %lld taken, %lld refused\n", accepted, refused);
    return 0;
}
