"""cgx_embed and cgx_embed_grad on the GPU against the formulas in 64 bits.

Tolerances follow from the arithmetic.  With u the unit roundoff of the type (2^-24, 2^-11, 2^-8):
  lookup    one product in binary32 (2^-24) and one rounding: (2^-24 + u) |exact|, and half a subnormal step of the type
  gradient  a binary32 sum of m terms, whatever its order (m 2^-24 of the sum of magnitudes), a product, an addition of what is
            there (2^-24 of each), one rounding (u |exact|)
"""
import math

import numpy as np
import pytest

from paper_2111_08617_amd import binding as cgx

pytestmark = pytest.mark.gpu

TYPES = {"f32": cgx.F32, "f16": cgx.F16, "bf16": cgx.BF16}
ROUNDOFF = {"f32": 2.0**-24, "f16": 2.0**-11, "bf16": 2.0**-8}
TINY = {"f32": 2.0**-126, "f16": 2.0**-25, "bf16": 2.0**-126}
GUARD = 64


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available(), "these tests need the MI355X"
    cgx.lib()
    return t


def dtype_of(torch, name):
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


def name_of(torch, dtype):
    return {torch.float32: "f32", torch.float16: "f16", torch.bfloat16: "bf16"}[dtype]


def guarded(torch, shape, dtype, value=-7.0):
    n = int(np.prod(shape))
    flat = torch.full((n + GUARD,), value, dtype=dtype, device="cuda")
    return flat[:n].view(shape), flat


def tokens_of(torch, n, vocab, kind, seed=0):
    g = torch.Generator().manual_seed(seed)
    if kind == "text":
        return (torch.rand(n, generator=g) ** 3 * vocab).long().clamp(max=vocab - 1)
    if kind == "one":
        return torch.full((n,), vocab // 2)
    if kind == "few":
        return torch.randint(0, min(vocab, 3), (n,), generator=g)
    if kind == "falling":
        return torch.arange(n).flip(0) % vocab
    return torch.randint(0, vocab, (n,), generator=g)


def look_up(torch, table, ids, scale=1.0, ignore=-100, stream=None):
    """The call's result; checked against the formula."""
    name = name_of(torch, table.dtype)
    out, flat = guarded(torch, (ids.numel(), table.shape[1]), table.dtype)
    cgx.cgx_embed(table, ids, out, scale=scale, ignore=ignore, stream=stream)
    torch.cuda.synchronize()
    assert (flat[-GUARD:] == -7.0).all(), "wrote past the output"
    counts, inside = ids != ignore, (ids >= 0) & (ids < table.shape[0])
    assert (out[~counts] == 0).all() and out[counts & ~inside].isnan().all()
    rows = counts & inside
    want = table[ids[rows]].double() * float(np.float32(scale))
    bound = (2.0**-24 + ROUNDOFF[name]) * want.abs() + TINY[name]
    assert ((out[rows].double() - want).abs() <= bound).all()
    return out


def gradient(torch, dout, ids, vocab, scale=1.0, ignore=-100, before=None, stream=None):
    """The call's result, added to `before` if that is given; checked against the formula."""
    name = name_of(torch, dout.dtype)
    (n, width), f = dout.shape, float(np.float32(scale))
    dtable, flat = guarded(torch, (vocab, width), dout.dtype)
    if before is not None:
        dtable.copy_(before)
    need = cgx.cgx_embed_grad_workspace(n, width, vocab, TYPES[name])
    ws = torch.full((need + 256,), 0xff, dtype=torch.uint8, device="cuda")
    cgx.cgx_embed_grad(dout, ids, dtable, ws[:need], scale=scale, ignore=ignore, accumulate=before is not None, stream=stream)
    torch.cuda.synchronize()
    assert (flat[-GUARD:] == -7.0).all(), "wrote past the table"
    assert (ws[need:] == 0xff).all(), "wrote past the workspace"
    rows = torch.nonzero((ids != ignore) & (ids >= 0) & (ids < vocab))[:, 0]
    want, size = (torch.zeros(vocab, width, dtype=torch.float64, device="cuda") for _ in range(2))
    for part in rows.split(4096):
        want.index_add_(0, ids[part], dout[part].double() * f)
        size.index_add_(0, ids[part], dout[part].double().abs() * abs(f))
    terms = torch.bincount(ids[rows], minlength=vocab)[:, None].double()
    total = want if before is None else want + before.double()
    bound = (terms + 2) * 2.0**-24 * size + (2.0**-23 + ROUNDOFF[name]) * total.abs() + TINY[name]
    assert ((dtable.double() - total).abs() <= bound).all()
    untouched = terms[:, 0] == 0
    if before is None:
        assert (dtable[untouched] == 0).all()
    else:
        assert torch.equal(dtable[untouched], before[untouched])
    return dtable


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(1, 1, 1), (1, 2048, 50257), (3, 5, 2), (17, 513, 300), (125, 519, 1003), (1000, 64, 70001), (2500, 1537, 400),
                                   (5000, 1030, 5000), (300, 8200, 129)], ids=lambda s: "x".join(map(str, s)))
def test_lookup(torch, shape, dtype):
    n, width, vocab = shape
    g = torch.Generator().manual_seed(n)
    table = torch.randn(vocab, width, generator=g).to(dtype_of(torch, dtype)).cuda()
    for scale in (1.0, math.sqrt(width), -0.3):
        look_up(torch, table, tokens_of(torch, n, vocab, "text", seed=width).cuda(), scale=scale)


@pytest.mark.parametrize("dtype", TYPES)
def test_lookup_of_padding_and_of_ids_outside(torch, dtype):
    table = torch.randn(50, 72).to(dtype_of(torch, dtype)).cuda()
    ids = torch.tensor([0, 49, 50, -1, -100, 7, 1 << 40, -(1 << 40), (1 << 32) + 3, 7, -100], device="cuda")
    look_up(torch, table, ids)
    look_up(torch, table, ids, ignore=7)                       # an entry of the vocabulary as padding
    look_up(torch, table, ids, ignore=1 << 40)
    look_up(torch, table, torch.zeros(0, dtype=torch.int64, device="cuda"))
    table[7] = float("inf")
    out = look_up(torch, table, torch.tensor([7, 8], device="cuda"), ignore=7)
    assert (out[0] == 0).all()


SHAPES = [(1, 1, 1), (1, 2048, 50257), (2, 3, 5), (7, 40, 3), (9, 513, 300), (64, 64, 64), (65, 72, 257), (125, 519, 1003), (1000, 96, 259),
          (4097, 136, 1000), (5000, 8, 100003), (20000, 24, 65537)]


@pytest.mark.parametrize("kind", ["text", "one", "few", "falling", "any"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_gradient(torch, shape, dtype, kind):
    n, width, vocab = shape
    g = torch.Generator().manual_seed(n)
    dout = (torch.randn(n, width, generator=g) + 0.25).to(dtype_of(torch, dtype)).cuda()
    ids = tokens_of(torch, n, vocab, kind, seed=width).cuda()
    gradient(torch, dout, ids, vocab, scale=0.7)
    before = torch.randn(vocab, width, generator=g).to(dout.dtype).cuda()
    gradient(torch, dout, ids, vocab, scale=-1.5, before=before)


@pytest.mark.parametrize("shape", [(70000, 64, 40), (33000, 520, 2000), (9000, 2048, 9000), (300, 2, (1 << 24) + 5), (200000, 1, 3)],
                         ids=lambda s: "x".join(map(str, s)))
def test_gradient_of_many_tokens_and_of_a_long_vocabulary(torch, shape):
    n, width, vocab = shape
    for dtype, kind in (("bf16", "text"), ("f32", "few"), ("f16", "any")):
        g = torch.Generator().manual_seed(n)
        dout = (torch.randn(n, width, generator=g) * 0.1).to(dtype_of(torch, dtype)).cuda()
        gradient(torch, dout, tokens_of(torch, n, vocab, kind, seed=5).cuda(), vocab)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("which", ["some", "first", "last", "all", "all but one", "most"])
def test_padding_takes_no_part_whatever_it_holds(torch, which, dtype):
    n, width, vocab = 500, 136, 90
    dout = torch.randn(n, width).to(dtype_of(torch, dtype)).cuda()
    ids = tokens_of(torch, n, vocab, "text").cuda()
    k = torch.arange(n, device="cuda")
    off = {"some": k % 3 == 1, "first": k < 330, "last": k >= 70, "all": k >= 0, "all but one": k != 77, "most": k % 40 != 0}[which]
    for mark, other in ((1 << 40, False), (5, False), (-100, True)):
        at = ids.clone()
        at[off] = mark
        if other:
            at[off] = torch.where(k[off] % 2 == 0, -1, vocab)        # outside the vocabulary: these have no row either
        rows = dout.clone()
        rows[at == mark] = float("nan")
        rows[(at < 0) | (at >= vocab)] = float("inf")
        gradient(torch, rows, at, vocab, ignore=mark)
        gradient(torch, rows, at, vocab, ignore=mark, before=torch.randn(vocab, width).to(dout.dtype).cuda())


def test_no_tokens(torch):
    for dtype in TYPES:
        for width, vocab in ((1, 1), (70, 300), (33, 65537)):
            dout = torch.zeros(0, width, dtype=dtype_of(torch, dtype), device="cuda")
            none = torch.zeros(0, dtype=torch.int64, device="cuda")
            gradient(torch, dout, none, vocab)
            gradient(torch, dout, none, vocab, before=torch.randn(vocab, width).to(dout.dtype).cuda())


def test_values_that_are_not_finite_stay_in_their_rows(torch):
    n, width, vocab = 300, 64, 20
    dout, ids = torch.randn(n, width, device="cuda"), tokens_of(torch, n, vocab, "any").cuda()
    dout[ids == 3, 5] = float("nan")
    dout[ids == 4, 6] = float("inf")
    dtable = torch.empty(vocab, width, device="cuda")
    ws = torch.empty(cgx.cgx_embed_grad_workspace(n, width, vocab, cgx.F32), dtype=torch.uint8, device="cuda")
    cgx.cgx_embed_grad(dout, ids, dtable, ws)
    bad = ~dtable.isfinite()
    assert bad[3, 5] and bad[4, 6] and bad.sum() == 2 and dtable[4, 6] == float("inf")


def test_the_gradient_is_the_lookups_adjoint(torch):
    """sum(out dout) = sum(table dtable) for any table, in small whole numbers, where every sum is exact."""
    n, width, vocab = 3000, 50, 211
    g = torch.Generator().manual_seed(1)
    table = torch.randint(-8, 9, (vocab, width), generator=g).float().cuda()
    dout = torch.randint(-8, 9, (n, width), generator=g).float().cuda()
    ids = tokens_of(torch, n, vocab, "text").cuda()
    ids[::7] = -100
    out = look_up(torch, table, ids, scale=2.0)
    dtable = gradient(torch, dout, ids, vocab, scale=2.0)
    assert float((out.double() * dout).sum()) == float((table.double() * dtable).sum())


def test_the_same_call_gives_the_same_bits(torch):
    n, width, vocab = 20000, 200, 300
    dout, ids = torch.randn(n, width, device="cuda").half(), tokens_of(torch, n, vocab, "text").cuda()
    first = gradient(torch, dout, ids, vocab)
    for _ in range(3):
        assert torch.equal(gradient(torch, dout, ids, vocab), first)


def test_ids_of_any_shape_and_tensors_that_start_anywhere_aligned(torch):
    table = torch.randn(100, 33, device="cuda")
    ids = torch.randint(0, 100, (6, 8), device="cuda")
    out = torch.empty(48, 33, device="cuda")
    cgx.cgx_embed(table, ids, out)
    assert torch.equal(out.view(6, 8, 33), table[ids])


def test_on_another_stream(torch):
    n, width, vocab = 4096, 256, 3000
    dout, ids = torch.randn(n, width, device="cuda"), tokens_of(torch, n, vocab, "text").cuda()
    table = torch.randn(vocab, width, device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    look_up(torch, table, ids, stream=s)
    want = gradient(torch, dout, ids, vocab, stream=s)
    with torch.cuda.stream(s):
        assert torch.equal(gradient(torch, dout, ids, vocab), want)


def test_two_calls_at_once_with_workspaces_of_their_own(torch):
    n, width, vocab = 8192, 512, 5000
    douts = [torch.randn(n, width, device="cuda") for _ in range(2)]
    ids = [tokens_of(torch, n, vocab, "text", seed=k).cuda() for k in range(2)]
    alone = [gradient(torch, d, i, vocab) for d, i in zip(douts, ids)]
    need = cgx.cgx_embed_grad_workspace(n, width, vocab, cgx.F32)
    ws = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(2)]
    out = [torch.empty(vocab, width, device="cuda") for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for k in range(2):
            cgx.cgx_embed_grad(douts[k], ids[k], out[k], ws[k], stream=streams[k])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, alone))


def test_captured_and_replayed(torch):
    n, width, vocab = 2000, 136, 700
    dout, ids = torch.randn(n, width, device="cuda").bfloat16(), tokens_of(torch, n, vocab, "text").cuda()
    table = torch.randn(vocab, width, device="cuda").bfloat16()
    out, dtable, total = torch.empty_like(dout), torch.empty_like(table), torch.zeros_like(table)
    ws = torch.empty(cgx.cgx_embed_grad_workspace(n, width, vocab, cgx.BF16), dtype=torch.uint8, device="cuda")

    def step():
        cgx.cgx_embed(table, ids, out, scale=2.0)
        cgx.cgx_embed_grad(dout, ids, dtable, ws, scale=2.0)
        cgx.cgx_embed_grad(dout, ids, total, ws, scale=2.0, accumulate=True)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        ids.copy_(tokens_of(torch, n, vocab, ("text", "one", "any", "few")[k], seed=k))
        dout.normal_()
        total.normal_()
        before = total.clone()
        dtable.fill_(5.0)
        ws.fill_(0xff)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, look_up(torch, table, ids, scale=2.0))
        assert torch.equal(dtable, gradient(torch, dout, ids, vocab, scale=2.0))
        assert torch.equal(total, gradient(torch, dout, ids, vocab, scale=2.0, before=before))


def test_a_tied_table_gets_both_its_gradients(torch):
    """The table is also the head's weight: lookup, head and both gradients into one buffer, against the formulas in 64 bits.  dweight and the sum are
    rounded to the type one after the other."""
    n, width, vocab = 300, 128, 1000
    for dtype in ("f32", "bf16"):
        table = (torch.randn(vocab, width, device="cuda") / 11).to(dtype_of(torch, dtype))
        ids = tokens_of(torch, n, vocab, "text").cuda()
        targets = torch.roll(ids, -1)
        targets[-1] = -100
        hidden = look_up(torch, table, ids, scale=3.0)
        ws = torch.empty(cgx.cgx_head_workspace(n, width, vocab, TYPES[dtype], True), dtype=torch.uint8, device="cuda")
        own = torch.empty(cgx.cgx_embed_grad_workspace(n, width, vocab, TYPES[dtype]), dtype=torch.uint8, device="cuda")
        loss, lse = torch.empty(2, n, device="cuda")
        dhidden, dtable = torch.empty_like(hidden), torch.empty_like(table)
        dloss = torch.full((n,), 1 / n, device="cuda")
        cgx.cgx_head_loss(hidden, table, targets, loss, lse, ws)
        cgx.cgx_head_loss_grad(hidden, table, targets, lse, dloss, dhidden, dtable, ws)
        head = dtable.clone()
        cgx.cgx_embed_grad(dhidden, ids, dtable, own, scale=3.0, accumulate=True)
        assert torch.equal(dtable, gradient(torch, dhidden, ids, vocab, scale=3.0, before=head))
        weight = table.cpu().double().requires_grad_()
        x = (weight[ids.cpu()] * 3.0).to(hidden.dtype).double() if dtype == "f32" else weight[ids.cpu()] * 3.0
        logp = torch.log_softmax(x @ weight.t(), dim=1)
        (-logp[torch.arange(n - 1), targets[:-1].cpu()].sum() / n).backward()
        off = float((dtable.cpu().double() - weight.grad).norm() / weight.grad.norm())
        # 2-norms; per element: hidden states, d, dhidden, dweight and their sum are rounded once each, every one by at most u of what it holds, and the
        # parts' norms are at most a few times the sum's
        assert off <= 5 * 4 * ROUNDOFF[dtype] + (1e-5 if dtype == "f32" else 0.0)


@pytest.mark.parametrize("vocab", [3, 700, 66000, 1 << 20])
def test_many_tokens_with_padding_and_ids_outside(torch, vocab):
    """Longer lists of tokens are cut into parts before they are sorted."""
    n, width = 40001, 40
    dout = torch.randn(n, width).bfloat16().cuda()
    ids = tokens_of(torch, n, vocab, "text", seed=3).cuda()
    k = torch.arange(n, device="cuda")
    ids[k % 11 == 3] = -100
    ids[k % 13 == 5] = vocab
    ids[k % 17 == 2] = (1 << 32) + 1
    ids[5000:9000] = -100
    dout[ids == -100] = float("nan")
    gradient(torch, dout, ids, vocab)
    gradient(torch, dout, ids, vocab, before=torch.randn(vocab, width).bfloat16().cuda())
    dout[ids == -100] = 0.5
    dout[ids == 1] = float("nan")
    gradient(torch, dout, ids, vocab, ignore=1)                # an entry of the vocabulary as padding


@pytest.mark.parametrize("tokens", [5, 300])
def test_the_longest_vocabulary(torch, tokens):
    """2^28 - 1 entries of one element: launches stay within their bounds, and every element is written."""
    vocab = (1 << 28) - 1
    g = torch.Generator().manual_seed(1)
    ids = torch.randint(0, vocab, (tokens,), generator=g).cuda()
    ids[0], ids[1], ids[2] = 0, vocab - 1, (1 << 27) + 1
    dout = torch.randint(1, 9, (tokens, 1), generator=g).bfloat16().cuda()
    dtable = torch.full((vocab, 1), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(cgx.cgx_embed_grad_workspace(tokens, 1, vocab, cgx.BF16), dtype=torch.uint8, device="cuda")
    cgx.cgx_embed_grad(dout, ids, dtable, ws)
    want = {}
    for k, v in zip(ids.tolist(), dout[:, 0].tolist()):
        want[k] = want.get(k, 0.0) + v
    at = torch.nonzero(dtable[:, 0])[:, 0]
    assert at.tolist() == sorted(want)
    assert dtable[at, 0].tolist() == [want[k] for k in sorted(want)]          # (whole numbers of at most 8 bits)
    out = torch.empty(tokens, 1, dtype=torch.bfloat16, device="cuda")
    cgx.cgx_embed(dtable, ids, out)
    assert out[:, 0].tolist() == [want[k] for k in ids.tolist()]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens", [3, 300])
def test_the_widest_rows(torch, tokens, dtype):
    g = torch.Generator().manual_seed(tokens)
    width, vocab = 1 << 17, 6
    ids = torch.randint(0, vocab, (tokens,), generator=g).cuda()
    table = torch.randn(vocab, width, generator=g).to(dtype_of(torch, dtype)).cuda()
    look_up(torch, table, ids, scale=0.5)
    dout = torch.randn(tokens, width, generator=g).to(table.dtype).cuda()
    gradient(torch, dout, ids, vocab)
    gradient(torch, dout, ids, vocab, before=table)
