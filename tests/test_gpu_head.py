"""cgx_head_loss and cgx_head_loss_grad on the GPU against the formulas in 64 bits.

Tolerances follow from the arithmetic.  With u the unit roundoff of the operands' type (2^-24, 2^-11, 2^-8):
  a logit is a binary32 sum of `width` products: |error| <= (width + 2) 2^-24 sum_h |x_h w_h| =: e
  lse: e of the logits; exp of a difference of up to 40 in binary32 (40 * 2^-23) and sums of at most 100 terms in a row
  (100 * 2^-24), together under 1.2e-5; and the rounding of the result, 2^-23 |lse|
  d: relative 2 e + 1.2e-5 of its probability, and u of itself where it is rounded to the operands' type (binary16: at least half
  a subnormal step under the scale, 2^-39 of the largest factor)
  its products: the same weighted by the other operand, binary32 sums of n terms (n 2^-24), and u of the result.
"""
import math

import numpy as np
import pytest

from paper_2111_08617_amd import binding as cgx

pytestmark = pytest.mark.gpu

TYPES = {"f32": cgx.F32, "f16": cgx.F16, "bf16": cgx.BF16}
ROUNDOFF = {"f32": 2.0**-24, "f16": 2.0**-11, "bf16": 2.0**-8}
GUARD = 64


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available(), "these tests need the MI355X"
    cgx.lib()
    return t


def dtype_of(torch, name):
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


def inputs(torch, tokens, width, vocab, dtype, seed=0, size=1.0):
    g = torch.Generator().manual_seed(seed)
    hidden = torch.randn(tokens, width, generator=g) * size
    weight = torch.randn(vocab, width, generator=g) / math.sqrt(width)
    targets = torch.randint(0, vocab, (tokens,), generator=g)
    dt = dtype_of(torch, dtype)
    return hidden.to(dt).cuda(), weight.to(dt).cuda(), targets.cuda()


def guarded(torch, shape, dtype):
    """(tensor of the shape filled with a value no result has, the flat buffer around it)."""
    n = int(np.prod(shape))
    flat = torch.full((n + GUARD,), -7.0, dtype=dtype, device="cuda")
    return flat[:n].view(shape), flat


def call(torch, hidden, weight, targets, dloss=None, ignore=-100, stream=None, slack=0):
    tokens, width = hidden.shape
    vocab = weight.shape[0]
    dt = {torch.float32: cgx.F32, torch.float16: cgx.F16, torch.bfloat16: cgx.BF16}[hidden.dtype]
    need = cgx.cgx_head_workspace(tokens, width, vocab, dt, dloss is not None)
    ws = torch.full((need + slack + 256,), 0xff, dtype=torch.uint8, device="cuda")     # NaN wherever it is read as a number
    loss, loss_all = guarded(torch, (tokens,), torch.float32)
    lse, lse_all = guarded(torch, (tokens,), torch.float32)
    cgx.cgx_head_loss(hidden, weight, targets, loss, lse, ws[:need], ignore=ignore, stream=stream)
    out = {"loss": loss, "lse": lse}
    guards = [loss_all, lse_all]
    if dloss is not None:
        out["dhidden"], a = guarded(torch, (tokens, width), hidden.dtype)
        out["dweight"], b = guarded(torch, (vocab, width), hidden.dtype)
        guards += [a, b]
        ws[:need].fill_(0xff)
        cgx.cgx_head_loss_grad(hidden, weight, targets, lse, dloss, out["dhidden"], out["dweight"], ws[:need], ignore=ignore, stream=stream)
    torch.cuda.synchronize()
    for g in guards:
        assert (g[-GUARD:] == -7.0).all(), "wrote past an output"
    assert (ws[need:] == 0xff).all(), "wrote past the workspace"
    return out


def check(torch, hidden, weight, targets, dloss=None, ignore=-100):
    """The calls' results against the formulas in 64 bits, within the bounds above."""
    got = call(torch, hidden, weight, targets, dloss, ignore)
    name = {torch.float32: "f32", torch.float16: "f16", torch.bfloat16: "bf16"}[hidden.dtype]
    u, width, vocab = ROUNDOFF[name], hidden.shape[1], weight.shape[0]
    counts = targets != ignore
    rows = torch.nonzero(counts)[:, 0]
    x, w, t = hidden[rows].double(), weight.double(), targets[rows]
    z = torch.mm(x, w.t())
    lse = torch.logsumexp(z, dim=1)
    loss = lse - z.gather(1, t[:, None])[:, 0]
    e = (width + 2) * 2.0**-24 * torch.mm(x.abs(), w.abs().t())
    top = e.max(dim=1).values if len(rows) else e.new_zeros(0)
    assert (got["loss"][~counts] == 0).all() and (got["lse"][~counts] == 0).all()
    bound = top + 1.2e-5 + 2.0**-23 * lse.abs()
    assert ((got["lse"][rows].double() - lse).abs() <= bound).all()
    assert ((got["loss"][rows].double() - loss).abs() <= bound + top + 2.0**-23 * loss.abs()).all()
    if dloss is None:
        return got
    takes = counts & (dloss != 0)
    assert (got["dhidden"][~takes] == 0).all()
    g = dloss[rows].double()[:, None]
    p = torch.exp(z - lse[:, None])
    d = g * p
    d[torch.arange(len(rows), device="cuda"), t] -= g[:, 0]
    kept = (dloss[rows] != 0)[:, None]
    d = torch.where(kept, d, 0.0)
    x = torch.where(kept, x, 0.0)
    smallest = 2.0**-39 * float(dloss.abs().max()) if name == "f16" and len(dloss) else 0.0
    off = g.abs() * p * (2 * e + 1.2e-5) + u * d.abs() + smallest
    off = torch.where(kept, off, 0.0)
    least = 2.0**-25 if name == "f16" else 1e-38
    dx, dw = torch.mm(d, w), torch.mm(d.t().contiguous(), x)
    bx = torch.mm(off + (vocab + 8) * 2.0**-24 * d.abs(), w.abs()) * 1.01 + u * dx.abs() + least
    bw = torch.mm((off + (len(rows) + 8) * 2.0**-24 * d.abs()).t().contiguous(), x.abs()) * 1.01 + u * dw.abs() + least
    assert ((got["dhidden"][rows].double() - dx).abs() <= bx).all()
    assert ((got["dweight"].double() - dw).abs() <= bw).all()
    return got


SHAPES = [(1, 1, 1), (1, 64, 2), (2, 3, 5), (1, 200, 1003), (17, 40, 129), (64, 64, 128), (65, 72, 257), (127, 129, 300), (128, 96, 511),
          (257, 519, 1003), (300, 256, 513)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_loss_and_gradients(torch, shape, dtype):
    hidden, weight, targets = inputs(torch, *shape, dtype, seed=sum(shape))
    g = torch.Generator().manual_seed(5)
    check(torch, hidden, weight, targets, torch.randn(shape[0], generator=g).cuda())


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("shape", [(512, 64, 25000), (6150, 2048, 300), (70, 2040, 6200), (1, 2048, 50257), (33, 768, 30522), (100, 1024, 20000)],
                         ids=lambda s: "x".join(map(str, s)))
def test_sizes_that_fill_the_chip(torch, shape, dtype):
    """Sides long enough for the large tiles, one side at a time; few tokens before a long vocabulary."""
    hidden, weight, targets = inputs(torch, *shape, dtype, seed=3)
    check(torch, hidden, weight, targets, torch.full((shape[0],), 1.0 / shape[0], device="cuda"))


@pytest.mark.parametrize("dtype", TYPES)
def test_a_vocabulary_in_several_pieces(torch, dtype):
    tokens, width, vocab = 16384, 24, 20011 if dtype == "f32" else 34001
    hidden, weight, targets = inputs(torch, tokens, width, vocab, dtype, seed=1, size=2.0)
    need = cgx.cgx_head_workspace(tokens, width, vocab, TYPES[dtype], True)
    assert need < tokens * vocab * (4 if dtype == "f32" else 2), "one piece: the test is about several"
    targets[::3] = -100
    check(torch, hidden, weight, targets, torch.full((tokens,), 0.25, device="cuda"))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("which", ["some", "first", "last", "all", "all but one", "most"])
def test_ignored_tokens_take_no_part_whatever_they_hold(torch, which, dtype):
    tokens, width, vocab = 200, 136, 700
    hidden, weight, targets = inputs(torch, tokens, width, vocab, dtype, seed=9)
    n = torch.arange(tokens, device="cuda")
    off = {"some": n % 3 == 1, "first": n < 130, "last": n >= 70, "all": n >= 0, "all but one": n != 77, "most": n % 40 != 0}[which]
    targets[off] = 1 << 40                                      # the mark is the caller's
    hidden[off] = torch.tensor([float("nan"), float("inf")], dtype=hidden.dtype, device="cuda").repeat(width // 2)
    got = check(torch, hidden, weight, targets, torch.full((tokens,), 0.5, device="cuda"), ignore=1 << 40)
    if which == "all":
        assert (got["dweight"] == 0).all() and (got["dhidden"] == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_tokens_with_no_weight_in_the_loss(torch, dtype):
    hidden, weight, targets = inputs(torch, 90, 64, 333, dtype, seed=4)
    dloss = torch.linspace(-1, 1, 90, device="cuda")
    dloss[10:70] = 0.0
    check(torch, hidden, weight, targets, dloss)
    # their hidden states have no influence on the gradients
    before = call(torch, hidden, weight, targets, dloss)
    hidden[10:70] = float("nan")
    after = call(torch, hidden, weight, targets, dloss)
    assert torch.equal(before["dweight"], after["dweight"]) and torch.equal(before["dhidden"], after["dhidden"])


@pytest.mark.parametrize("dtype", TYPES)
def test_targets_outside_the_vocabulary_are_not_silent(torch, dtype):
    hidden, weight, targets = inputs(torch, 40, 64, 300, dtype)
    targets[7], targets[9] = 300, -5
    got = call(torch, hidden, weight, targets, torch.ones(40, device="cuda"))
    bad = torch.zeros(40, dtype=torch.bool, device="cuda")
    bad[[7, 9]] = True
    assert got["loss"][bad].isnan().all() and got["loss"][~bad].isfinite().all()
    assert got["dhidden"][bad].isnan().all() and got["dhidden"][~bad].isfinite().all()
    assert got["dweight"].isnan().all()


def test_no_tokens_leave_a_zero_gradient(torch):
    for dtype in TYPES:
        hidden, weight, targets = inputs(torch, 0, 70, 300, dtype)
        got = call(torch, hidden, weight, targets, torch.zeros(0, device="cuda"))
        assert (got["dweight"] == 0).all()


@pytest.mark.parametrize("scale", [2.0**-20, 1.0, 65536.0])
def test_loss_scales_and_uneven_factors_in_binary16(torch, scale):
    """Probabilities around 1e-4 under factors from 1e-3 to 1: far below the smallest binary16 number unless d is scaled."""
    hidden, weight, targets = inputs(torch, 140, 128, 9000, "f16", seed=8)
    dloss = scale * torch.logspace(-3, 0, 140, device="cuda") / 64
    check(torch, hidden, weight * 0.125 if scale > 1 else weight, targets, dloss)


@pytest.mark.parametrize("dtype", TYPES)
def test_large_logits(torch, dtype):
    """Logits of several hundred: exp of them overflows, and most probabilities underflow."""
    hidden, weight, targets = inputs(torch, 60, 64, 500, dtype, seed=2, size=100.0)
    check(torch, hidden, weight, targets, torch.ones(60, device="cuda"))


def test_gradients_against_differences(torch):
    """Directional derivatives of the loss in 64 bits by central differences: truncation around 1e-9 at this step."""
    hidden, weight, targets = inputs(torch, 37, 50, 210, "f32", seed=6)
    dloss = torch.linspace(-1, 2, 37, device="cuda")
    got = call(torch, hidden, weight, targets, dloss)

    def value(x, w):
        z = torch.mm(x, w.t())
        return (dloss.double() * (torch.logsumexp(z, dim=1) - z.gather(1, targets[:, None])[:, 0])).sum()

    x, w, step = hidden.double(), weight.double(), 1e-5
    g = torch.Generator(device="cuda").manual_seed(1)
    for _ in range(8):
        a, b = (torch.randn(t.shape, dtype=torch.float64, device="cuda", generator=g) for t in (x, w))
        by_x = (value(x + step * a, w) - value(x - step * a, w)) / (2 * step)
        by_w = (value(x, w + step * b) - value(x, w - step * b)) / (2 * step)
        assert abs(float((got["dhidden"].double() * a).sum() - by_x)) <= 1e-5 * float((got["dhidden"].double() * a).abs().sum())
        assert abs(float((got["dweight"].double() * b).sum() - by_w)) <= 1e-5 * float((got["dweight"].double() * b).abs().sum())


@pytest.mark.parametrize("dtype", TYPES)
def test_same_call_same_bits_and_other_streams(torch, dtype):
    hidden, weight, targets = inputs(torch, 700, 128, 2100, dtype, seed=12)
    dloss = torch.full((700,), 1 / 700.0, device="cuda")
    first = call(torch, hidden, weight, targets, dloss)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = call(torch, hidden, weight, targets, dloss)
    third = call(torch, hidden, weight, targets, dloss, stream=side)
    for k, v in first.items():
        assert torch.equal(v, second[k]) and torch.equal(v, third[k]), k


def test_captured_into_a_graph(torch):
    hidden, weight, targets = inputs(torch, 300, 192, 1500, "bf16", seed=13)
    dloss = torch.full((300,), 1 / 300.0, device="cuda")
    ws = torch.empty(cgx.cgx_head_workspace(300, 192, 1500, cgx.BF16, True), dtype=torch.uint8, device="cuda")
    loss, lse = torch.empty(300, device="cuda"), torch.empty(300, device="cuda")
    dh, dw = torch.empty_like(hidden), torch.empty_like(weight)

    def step():
        cgx.cgx_head_loss(hidden, weight, targets, loss, lse, ws)
        cgx.cgx_head_loss_grad(hidden, weight, targets, lse, dloss, dh, dw, ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        hidden.copy_(inputs(torch, 300, 192, 1500, "bf16", seed=40 + k)[0])
        targets[k::7] = -100
        want = {n: t.clone() for n, t in call(torch, hidden, weight, targets, dloss).items()}
        for t in (loss, lse, dh, dw):
            t.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, want["loss"]) and torch.equal(lse, want["lse"])
        assert torch.equal(dh, want["dhidden"]) and torch.equal(dw, want["dweight"])


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("tokens", [447, 448, 449, 480, 512, 513, 1100])
def test_the_last_round_of_the_weights_tiles(torch, tokens, dtype):
    """260 tiles of the weight's gradient: four more than the chip takes at once, split over the tokens where these are enough."""
    hidden, weight, targets = inputs(torch, tokens, 1024, 16640 - 3, dtype, seed=tokens)
    targets[5::9] = -100
    check(torch, hidden, weight, targets, torch.full((tokens,), 1.0 / tokens, device="cuda"))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("tokens", [8, 30, 100, 1000])
def test_a_means_factor_is_not_rounded_in_every_target(torch, tokens, dtype):
    """1 / tokens is no number of 16 bits.  Were d rounded in units of 1, every target of a call would be off by the same 2^-9 (2^-12) or so,
    and the gradients of tokens that a model knows nothing of with them.  A target at probability p is -(1 - p) in units of the factor:
    stored as -1, off by p, where p is below half a unit roundoff (here about 1 / vocab); the other elements of d, each off by up to u of
    itself and in no common direction, hold 1 / sqrt(vocab) of its size.  So a gradient is hardly further from the exact one than that one
    rounded to its type."""
    vocab, width = 20000, 256
    hidden, weight, targets = inputs(torch, tokens, width, vocab, dtype, seed=17, size=0.05)
    got = call(torch, hidden, weight, targets, torch.full((tokens,), 1.0 / tokens, device="cuda"))
    x, w = hidden.double(), weight.double()
    d = torch.softmax(torch.mm(x, w.t()), dim=1)
    d[torch.arange(tokens, device="cuda"), targets] -= 1.0
    for name, want in (("dhidden", torch.mm(d, w) / tokens), ("dweight", torch.mm(d.t().contiguous(), x) / tokens)):
        off, rounded = (float((t.double() - want).norm() / want.norm()) for t in (got[name], want.to(hidden.dtype)))
        assert off <= rounded + 2.0 / vocab + 0.05 * ROUNDOFF[dtype], (name, off, rounded)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", [64, 128, 192, 320, 1088])
@pytest.mark.parametrize("tokens", [1, 15, 16, 17, 33, 64])
def test_few_tokens_at_the_ends_of_tiles_and_quarters(torch, tokens, width, dtype):
    # widths of 1 to 17 units of 128 bytes (2 to 34 for f32): quarters that are empty, odd, uneven
    for vocab in (1, 31, 33, 64, 1003):
        hidden, weight, targets = inputs(torch, tokens, width, vocab, dtype, seed=tokens + width + vocab)
        targets[tokens // 2] = -100 if tokens > 1 else targets[0]
        check(torch, hidden, weight, targets)


@pytest.mark.parametrize("tokens", [2, 20])
def test_few_tokens_over_more_parts_than_one_pass_joins(torch, tokens):
    # 16 waves of a token's block take 4096 parts at a time: 131072 columns in blocks of 32, 262144 in tiles of 64
    hidden, weight, targets = inputs(torch, tokens, 64, 300007, "bf16", seed=3)
    targets[0], targets[1] = 300006, 262144
    check(torch, hidden, weight, targets)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens", [7, 40])
def test_a_tokens_nan_and_infinity_stay_its_own(torch, tokens, dtype):
    hidden, weight, targets = inputs(torch, tokens, 256, 500, dtype, seed=tokens)
    targets[2] = -100
    clean = call(torch, hidden, weight, targets)
    bad = hidden.clone()
    bad[2, 5] = math.nan                                 # of a token that does not count
    bad[4, 200] = math.nan
    bad[5, 0] = math.inf
    got = call(torch, bad, weight, targets)
    assert torch.isnan(got["loss"][4]) and torch.isnan(got["loss"][5])
    keep = [k for k in range(tokens) if k not in (4, 5)]
    assert torch.equal(got["loss"][keep], clean["loss"][keep]) and torch.equal(got["lse"][keep], clean["lse"][keep])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", [1, 7, 31, 33, 63, 65, 72, 127, 129, 321, 1766])
def test_few_tokens_of_any_width(torch, width, dtype):
    # rows that start at any element, with a last unit of every kind; nothing past the weight's end is read (its last row ends an allocation's use)
    for tokens, vocab in ((1, 1), (3, 65), (16, 130), (17, 33), (50, 97), (64, 31)):
        hidden, weight, targets = inputs(torch, tokens, width, vocab, dtype, seed=tokens + width)
        check(torch, hidden, weight, targets)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(65, 96, 1), (256, 1024, 1000), (257, 130, 769), (1000, 66, 255), (4096, 64, 64), (4097, 64, 64), (100, 519, 2000)],
                         ids=lambda s: "x".join(map(str, s)))
def test_few_logits_of_many_tokens(torch, shape, dtype):
    hidden, weight, targets = inputs(torch, *shape, dtype, seed=sum(shape))
    targets[1::3] = -100
    hidden[4] = math.nan                                 # (4 = 1 + 3: does not count)
    check(torch, hidden, weight, targets)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("size", [1.0, 100.0, 1e-30])
def test_a_factor_that_is_not_finite_stays_its_tokens(torch, size, bad, dtype):
    """dhidden of a token depends on its own factor: those of the others are the same as where the token takes no part, in every bit,
    as the units of d come from the finite factors either way.  (dweight is a sum over all tokens and is not finite by the formula.)"""
    tokens, at = 90, 41
    hidden, weight, targets = inputs(torch, tokens, 64, 333, dtype, seed=21)
    dloss = torch.linspace(-size, size, tokens, device="cuda")
    others = torch.arange(tokens, device="cuda") != at
    dloss[at] = 0.0
    want = check(torch, hidden, weight, targets, dloss)
    dloss[at] = bad
    got = call(torch, hidden, weight, targets, dloss)
    assert torch.equal(got["dhidden"][others], want["dhidden"][others])
    assert not got["dhidden"][at].isfinite().any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("counts", ["all", "two in three"])
@pytest.mark.parametrize("width", [24, 64, 192])
def test_several_pieces_of_weights_as_they_lie_and_of_padded_ones(torch, width, counts, dtype):
    """Rows of whole steps are read where they lie, piece by piece; hidden states too where every token counts and the tokens are whole steps."""
    tokens, vocab = 16384, 20011 if dtype == "f32" else 34001
    size = 4 if dtype == "f32" else 2
    hidden, weight, targets = inputs(torch, tokens, width, vocab, dtype, seed=width)
    # a piece has a multiple of 256 columns: d of two pieces would not fit the workspace, and no such number divides the vocabulary
    need = cgx.cgx_head_workspace(tokens, width, vocab, TYPES[dtype], True)
    assert need < tokens * vocab * size and vocab % 256
    targets[0], targets[1], targets[2] = vocab - 1, 0, vocab // 2
    if counts != "all":
        targets[::3] = -100
    check(torch, hidden, weight, targets, torch.linspace(-1.0, 1.0, tokens, device="cuda"))
