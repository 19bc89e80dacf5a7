"""cgx_head_distill and cgx_head_distill_grad on the GPU against the formulas in 64 bits.

Tolerances follow from the arithmetic.  With u the unit roundoff of the operands' type (2^-24, 2^-11, 2^-8), T the temperature:
  a logit z is a binary32 sum of `width` products: |error| <= (width + 2) 2^-24 sum_h |x_h w_h| =: e; so is picked
  lse: e / T of the logits, their product with 1 / T (2 2^-24 |z| / T); exp of a difference of up to 40 in binary32 (40 * 2^-23) and sums of at
  most 100 terms in a row (100 * 2^-24), together under 1.2e-5; and the rounding of the result, 2^-23 |lse|
  q: relative, exp of a difference (2^-23 and 2^-23 of the magnitudes in it) and a sum of at most 1024 terms in 64 lanes (22 * 2^-24)
  loss: those of q, of lse and of picked in its terms, the terms' own roundings (2^-22 of the magnitudes in them), sums of `entries` terms
  d: relative (e / T + 2^-23 |z| / T, of the logit and of the row's largest) + 1.2e-5 + 2^-23 |lse| of its probability, q's error, 2^-23 of both for the difference, and u of
  itself where it is rounded to the operands' type or a finer one (binary16, which also holds that of many bfloat16 tokens: at least half a
  subnormal step under the scale, 2^-39 of the largest factor)
  operands in binary16 instead of bfloat16: half a subnormal step under their power of two, 2^-25 / 2^3 of the largest magnitude
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


def name_of(torch, dtype):
    return {torch.float32: "f32", torch.float16: "f16", torch.bfloat16: "bf16"}[dtype]


def inputs(torch, tokens, width, vocab, entries, dtype, teacher="f32", seed=0, size=1.0, marked=0.2):
    """Entries may come twice in a row, as they do where the vocabulary is short."""
    g = torch.Generator().manual_seed(seed)
    hidden = torch.randn(tokens, width, generator=g) * size
    weight = torch.randn(vocab, width, generator=g) / math.sqrt(width)
    ids = torch.randint(0, vocab, (tokens, entries), generator=g)
    logits = torch.randn(tokens, entries, generator=g) * 3 + 5
    ids[torch.rand(tokens, entries, generator=g) < marked] = -100
    dt = dtype_of(torch, dtype)
    return hidden.to(dt).cuda(), weight.to(dt).cuda(), ids.cuda(), logits.to(dtype_of(torch, teacher)).cuda()


def guarded(torch, shape, dtype):
    n = int(np.prod(shape))
    flat = torch.full((n + GUARD,), -7.0, dtype=dtype, device="cuda")
    return flat[:n].view(shape), flat


def call(torch, hidden, weight, ids, teacher, dloss=None, temperature=1.0, ignore=-100, stream=None):
    (tokens, width), vocab, entries = hidden.shape, weight.shape[0], ids.shape[1]
    dt = TYPES[name_of(torch, hidden.dtype)]
    need = cgx.cgx_head_distill_workspace(tokens, width, vocab, entries, dt, dloss is not None)
    ws = torch.full((need + 256,), 0xff, dtype=torch.uint8, device="cuda")            # NaN wherever it is read as a number
    out, guards = {}, []
    for what, shape in (("loss", (tokens,)), ("lse", (tokens,)), ("picked", (tokens, entries))):
        out[what], flat = guarded(torch, shape, torch.float32)
        guards.append(flat)
    cgx.cgx_head_distill(hidden, weight, ids, teacher, out["loss"], out["lse"], out["picked"], ws[:need], temperature=temperature, ignore=ignore,
                         stream=stream)
    if dloss is not None:
        for what, shape in (("dhidden", (tokens, width)), ("dweight", (vocab, width))):
            out[what], flat = guarded(torch, shape, hidden.dtype)
            guards.append(flat)
        if stream is None:
            ws[:need].fill_(0xff)
        cgx.cgx_head_distill_grad(hidden, weight, ids, teacher, out["lse"], out["picked"], dloss, out["dhidden"], out["dweight"], ws[:need],
                                  temperature=temperature, ignore=ignore, stream=stream)
    torch.cuda.synchronize()
    assert all((g[-GUARD:] == -7.0).all() for g in guards), "wrote past an output"
    assert (ws[need:] == 0xff).all(), "wrote past the workspace"
    return out


def check(torch, hidden, weight, ids, teacher, dloss=None, temperature=1.0, ignore=-100):
    """The calls' results against the formulas in 64 bits, within the bounds above.  Ids are inside the vocabulary or marked."""
    got = call(torch, hidden, weight, ids, teacher, dloss, temperature, ignore)
    name = name_of(torch, hidden.dtype)
    u, (tokens, width), vocab, entries, t = ROUNDOFF[name], hidden.shape, weight.shape[0], ids.shape[1], float(np.float32(temperature))
    there = ids != ignore
    soft = torch.where(there, teacher.double(), -math.inf) / t
    takes = (soft > -math.inf).any(dim=1)
    for what in ("loss", "lse", "picked"):
        assert (got[what][~takes] == 0).all()
    assert (got["picked"][~there] == 0).all()
    rows = torch.nonzero(takes)[:, 0]
    x, w, there, soft = hidden[rows].double(), weight.double(), there[rows], soft[rows]
    at = torch.where(there, ids[rows], 0)
    z = torch.mm(x, w.t())
    e = (width + 2) * 2.0**-24 * torch.mm(x.abs(), w.abs().t())
    picked = torch.where(there, z.gather(1, at), 0.0)
    assert ((got["picked"][rows].double() - picked).abs() <= torch.where(there, e.gather(1, at), 0.0)).all()
    lse = torch.logsumexp(z / t, dim=1, keepdim=True)
    off_z = e / t + 2.0**-23 * z.abs() / t
    off_lse = (off_z.max(dim=1, keepdim=True).values if len(rows) else off_z[:, :1]) + 1.2e-5 + 2.0**-23 * lse.abs()
    assert ((got["lse"][rows, None].double() - lse).abs() <= off_lse).all()
    top = soft.max(dim=1, keepdim=True).values if len(rows) else soft[:, :1]
    q = torch.softmax(soft, dim=1)
    mass = torch.logsumexp(soft, dim=1, keepdim=True)
    size = torch.where(q > 0, soft.abs(), 0.0)
    off_q = 2.0**-23 * (1 + size + top.abs() + (size - top.abs()).abs()) + 22 * 2.0**-24 + 2.0**-23
    term = torch.where(q > 0, torch.where(q > 0, soft, 0.0) - mass + lse - picked / t, 0.0)
    loss = (q * term).sum(dim=1)
    off = q * (off_q * term.abs() + off_lse + torch.where(there, off_z.gather(1, at), 0.0) + 2.0**-23 * (1 + mass.abs()) +
               2.0**-22 * (size + mass.abs() + lse.abs() + picked.abs() / t)) + entries * 2.0**-24 * q * term.abs()
    assert ((got["loss"][rows].double() - loss).abs() <= off.sum(dim=1) + 2.0**-23 * loss.abs()).all()
    if dloss is None:
        return got
    kept = dloss != 0
    assert (got["dhidden"][~(takes & kept)] == 0).all()
    kept = kept[rows][:, None]
    g = torch.where(kept, dloss[rows].double()[:, None], 0.0)
    p = torch.exp(z / t - lse)
    at_entries, off_entries = torch.zeros_like(p).scatter_add_(1, at, q), torch.zeros_like(p).scatter_add_(1, at, q * off_q)
    d = g * (p - at_entries)
    x = torch.where(kept, x, 0.0)
    smallest = 2.0**-39 * float(dloss.abs().max()) if name != "f32" and len(dloss) else 0.0
    step = 2.0**-28 if name == "bf16" else 0.0
    # (a logit's own error, and that of lse, which is the largest logit's at most)
    of_p = off_z + (off_z.max(dim=1, keepdim=True).values if len(rows) else off_z[:, :1])
    off = g.abs() * (p * (of_p + 1.2e-5 + 2.0**-22 * (1 + lse.abs())) + off_entries + 2.0**-23 * (p + at_entries)) * 1.01 + u * d.abs() + smallest
    off = torch.where(kept, off, 0.0)
    least = 2.0**-25 if name == "f16" else 1e-38
    dx, dw = torch.mm(d, w) / t, torch.mm(d.t().contiguous(), x) / t
    bx = torch.mm(off + (vocab + 8) * 2.0**-24 * d.abs(), w.abs() + step * w.abs().max()) * 1.01 / t + step * d.abs().sum(dim=1, keepdim=True) * w.abs().max() / t + (u + 2.0**-22) * dx.abs() + least
    bw = torch.mm((off + (len(rows) + 8) * 2.0**-24 * d.abs()).t().contiguous(), x.abs()) * 1.01 / t + (step * x.abs().max() * d.abs().sum(dim=0)[:, None] / t if len(rows) else 0.0) + (u + 2.0**-22) * dw.abs() + least
    assert ((got["dhidden"][rows].double() - dx).abs() <= bx).all()
    assert ((got["dweight"].double() - dw).abs() <= bw).all()
    return got


SHAPES = [(1, 1, 1, 1), (1, 64, 2, 5), (2, 3, 5, 3), (1, 200, 1003, 17), (17, 40, 129, 64), (64, 64, 128, 65), (65, 72, 257, 1), (127, 129, 300, 33),
          (128, 96, 511, 130), (257, 519, 1003, 40), (300, 256, 513, 9), (5, 64, 50, 1024)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_divergence_and_gradients(torch, shape, dtype):
    args = inputs(torch, *shape, dtype, seed=sum(shape), teacher=("f32", "f16", "bf16")[shape[1] % 3])
    g = torch.Generator().manual_seed(5)
    check(torch, *args, torch.randn(shape[0], generator=g).cuda(), temperature=(1.0, 2.0, 0.7)[shape[0] % 3])


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("shape", [(512, 64, 25000, 64), (6150, 2048, 300, 20), (70, 2040, 6200, 256), (1, 2048, 50257, 64), (33, 768, 30522, 32),
                                   (100, 1024, 20000, 1000), (3000, 64, 5000, 128), (40, 64, 8000, 1000)], ids=lambda s: "x".join(map(str, s)))
def test_sizes_that_fill_the_chip(torch, shape, dtype):
    check(torch, *inputs(torch, *shape, dtype, seed=3), torch.full((shape[0],), 1.0 / shape[0], device="cuda"), temperature=1.5)


@pytest.mark.parametrize("dtype", TYPES)
def test_a_vocabulary_in_several_pieces(torch, dtype):
    tokens, width, vocab = 16384, 24, 20011 if dtype == "f32" else 34001
    args = inputs(torch, tokens, width, vocab, 12, dtype, seed=1, size=2.0)
    need = cgx.cgx_head_distill_workspace(tokens, width, vocab, 12, TYPES[dtype], True)
    assert need < tokens * vocab * (4 if dtype == "f32" else 2), "one piece: the test is about several"
    args[2][::3] = -100
    check(torch, *args, torch.full((tokens,), 0.25, device="cuda"))


@pytest.mark.parametrize("temperature", [2.0**-10, 0.25, 1.0, 8.0, 100.0, 2.0**10])
@pytest.mark.parametrize("dtype", TYPES)
def test_temperatures(torch, dtype, temperature):
    check(torch, *inputs(torch, 90, 64, 700, 30, dtype, seed=2), torch.linspace(-1, 1, 90, device="cuda"), temperature=temperature)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("which", ["some", "first", "last", "all", "all but one", "most"])
def test_tokens_without_entries_take_no_part_whatever_they_hold(torch, which, dtype):
    tokens, width, vocab = 200, 136, 700
    hidden, weight, ids, teacher = inputs(torch, tokens, width, vocab, 6, dtype, seed=9, marked=0.0)
    n = torch.arange(tokens, device="cuda")
    off = {"some": n % 3 == 1, "first": n < 130, "last": n >= 70, "all": n >= 0, "all but one": n != 77, "most": n % 40 != 0}[which]
    ids[off] = 1 << 40                                          # the mark is the caller's
    teacher[off] = float("nan")
    hidden[off] = torch.tensor([float("nan"), float("inf")], dtype=hidden.dtype, device="cuda").repeat(width // 2)
    half = off & (n % 2 == 0)
    ids[half] = 3                                               # entries of no share at all are no entries either
    teacher[half] = float("-inf")
    args = [torch.where(off[:, None], 0.0, hidden.float()).to(hidden.dtype), weight, ids, teacher]
    dloss = torch.full((tokens,), 0.5, device="cuda")
    want = check(torch, *args, dloss, ignore=1 << 40)
    got = call(torch, hidden, weight, ids, teacher, dloss, ignore=1 << 40)
    assert all(torch.equal(got[k], want[k]) for k in want)
    if which == "all":
        assert (got["dweight"] == 0).all() and (got["dhidden"] == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens", [12, 150])
def test_repeated_and_vanishing_entries(torch, dtype, tokens):
    """The same id in every place, twice, and beside entries with a share of 0."""
    hidden, weight, ids, teacher = inputs(torch, tokens, 72, 300, 70, dtype, seed=6)
    ids[0] = 5
    ids[1, 1:] = ids[1, :-1].clone()
    ids[2, ::2] = 299
    teacher[3, :69] = float("-inf")
    ids[3, 69] = 7
    teacher[4, 3:] = -1e4
    ids[4, :3] = torch.tensor([8, 9, 8], device="cuda")
    check(torch, hidden, weight, ids, teacher, torch.ones(tokens, device="cuda"))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens", [40, 130])
def test_what_is_wrong_is_not_silent(torch, dtype, tokens):
    hidden, weight, ids, teacher = inputs(torch, tokens, 64, 300, 20, dtype, marked=0.0)
    ids[7, 3], ids[9, 19], ids[11, 0] = 300, -5, (1 << 32) + 4
    teacher[13, 2], teacher[15, 0] = float("nan"), float("inf")
    teacher[7] = float("-inf")
    got = call(torch, hidden, weight, ids, teacher, torch.ones(tokens, device="cuda"))
    bad = torch.zeros(tokens, dtype=torch.bool, device="cuda")
    bad[[7, 9, 11, 13, 15]] = True
    assert got["loss"][bad].isnan().all() and got["loss"][~bad].isfinite().all()
    assert got["dhidden"][bad].isnan().all() and got["dhidden"][~bad].isfinite().all()
    assert got["dweight"].isnan().all()
    assert got["picked"].isnan().sum() == 3 and got["lse"].isfinite().all()
    # without a weight in the step's loss they take no part in its gradients
    dloss = torch.where(bad, 0.0, 1.0)
    got = call(torch, hidden, weight, ids, teacher, dloss)
    assert (got["dhidden"][bad] == 0).all() and got["dweight"].isfinite().all()


@pytest.mark.parametrize("dtype", TYPES)
def test_logits_that_are_not_finite(torch, dtype):
    hidden, weight, ids, teacher = inputs(torch, 100, 64, 300, 8, dtype, marked=0.0)
    hidden[3, 5], hidden[4, 6] = float("nan"), float("inf")
    got = call(torch, hidden, weight, ids, teacher)
    for what in ("loss", "lse"):
        assert got[what][3:5].isnan().all() and got[what][:3].isfinite().all() and got[what][5:].isfinite().all()


def test_no_tokens_leave_a_zero_gradient(torch):
    for dtype in TYPES:
        got = call(torch, *inputs(torch, 0, 70, 300, 4, dtype), torch.zeros(0, device="cuda"))
        assert (got["dweight"] == 0).all()


@pytest.mark.parametrize("scale", [2.0**-20, 1.0, 65536.0])
def test_loss_scales_and_uneven_factors_in_binary16(torch, scale):
    hidden, weight, ids, teacher = inputs(torch, 140, 128, 9000, 50, "f16", seed=8)
    dloss = scale * torch.logspace(-3, 0, 140, device="cuda") / 64
    check(torch, hidden, weight * 0.125 if scale > 1 else weight, ids, teacher, dloss)


def test_one_entry_is_the_loss_of_a_target(torch):
    """A teacher that is certain: cgx_head_loss and its gradients.  The tiles are the same; the target's logit is summed in another order here,
    2 (width + 2) 2^-24 sum |x w| apart at most, and its d by that and a rounding."""
    for dtype in TYPES:
        for tokens in (20, 300):
            hidden, weight, ids, teacher = inputs(torch, tokens, 136, 900, 1, dtype, seed=4)
            got = call(torch, hidden, weight, ids, teacher, torch.ones(tokens, device="cuda"))
            ws = torch.empty(cgx.cgx_head_workspace(tokens, 136, 900, TYPES[dtype], True), dtype=torch.uint8, device="cuda")
            loss, lse = torch.empty(2, tokens, device="cuda")
            dhidden, dweight = torch.empty_like(hidden), torch.empty_like(weight)
            targets = ids[:, 0].contiguous()
            cgx.cgx_head_loss(hidden, weight, targets, loss, lse, ws)
            cgx.cgx_head_loss_grad(hidden, weight, targets, lse, torch.ones(tokens, device="cuda"), dhidden, dweight, ws)
            e = 2 * 138 * 2.0**-24 * (hidden.float().abs() * weight.float().abs()[targets.clamp(min=0)]).sum(dim=1)
            assert torch.equal(lse, got["lse"])
            assert ((loss - got["loss"]).abs() <= e + 2.0**-22 * (lse.abs() + loss.abs() + 1)).all()
            for a, b in ((dhidden, got["dhidden"]), (dweight, got["dweight"])):
                # another rounding of a row's target, and of the results: 2 u of each, and what e changes in a probability
                assert float((a.double() - b.double()).norm()) <= (4 * ROUNDOFF[dtype] + 2 * float(e.max()) + 2.0**-20) * float(a.double().norm())


def test_gradients_against_differences(torch):
    """Central differences of the loss in binary32: 1e-2 apart, so that its rounding (1e-6 here) stays below 1e-4 of them; the third
    derivative's part is under 1e-4 for hidden states and weights of this size."""
    hidden, weight, ids, teacher = inputs(torch, 6, 12, 30, 4, "f32", seed=12)
    dloss = torch.linspace(0.5, 1.5, 6, device="cuda")
    got = call(torch, hidden, weight, ids, teacher, dloss, temperature=2.0)
    h = 1e-2

    def value():
        return float((call(torch, hidden, weight, ids, teacher, temperature=2.0)["loss"].double() * dloss).sum())

    for tensor, grad in ((hidden, got["dhidden"]), (weight, got["dweight"])):
        for k in range(0, tensor.numel(), 7):
            flat, before = tensor.view(-1), float(tensor.view(-1)[k])
            flat[k] = before + h
            up, there = value(), float(flat[k])
            flat[k] = before - h
            down, back = value(), float(flat[k])
            flat[k] = before
            assert abs((up - down) / (there - back) - float(grad.view(-1)[k])) < 1e-3


def test_the_same_call_gives_the_same_bits(torch):
    args = inputs(torch, 700, 256, 3000, 40, "bf16", seed=7)
    dloss = torch.ones(700, device="cuda")
    first = call(torch, *args, dloss)
    for _ in range(3):
        again = call(torch, *args, dloss)
        assert all(torch.equal(first[k], again[k]) for k in first)


def test_on_another_stream(torch):
    args = inputs(torch, 300, 128, 2000, 16, "bf16", seed=7)
    dloss = torch.ones(300, device="cuda")
    want = call(torch, *args, dloss)
    s = torch.cuda.Stream()
    got = call(torch, *args, dloss, stream=s)
    assert all(torch.equal(want[k], got[k]) for k in want)


@pytest.mark.parametrize("tokens", [4, 200])
def test_captured_and_replayed(torch, tokens):
    width, vocab, entries = 136, 900, 24
    hidden, weight, ids, teacher = inputs(torch, tokens, width, vocab, entries, "f16")
    loss, lse = torch.empty(2, tokens, device="cuda")
    picked, dloss = torch.empty(tokens, entries, device="cuda"), torch.ones(tokens, device="cuda")
    dhidden, dweight = torch.empty_like(hidden), torch.empty_like(weight)
    ws = torch.empty(cgx.cgx_head_distill_workspace(tokens, width, vocab, entries, cgx.F16, True), dtype=torch.uint8, device="cuda")

    def step():
        cgx.cgx_head_distill(hidden, weight, ids, teacher, loss, lse, picked, ws, temperature=3.0)
        cgx.cgx_head_distill_grad(hidden, weight, ids, teacher, lse, picked, dloss, dhidden, dweight, ws, temperature=3.0)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        new = inputs(torch, tokens, width, vocab, entries, "f16", teacher="f32", seed=20 + k, marked=(0.0, 0.3, 0.9, 1.0)[k])
        for a, b in zip((hidden, weight, ids, teacher), new):
            a.copy_(b)
        ws.fill_(0xff)
        graph.replay()
        torch.cuda.synchronize()
        want = call(torch, hidden, weight, ids, teacher, dloss, temperature=3.0)
        for what, t in (("loss", loss), ("lse", lse), ("picked", picked), ("dhidden", dhidden), ("dweight", dweight)):
            assert torch.equal(t, want[what]), what


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("tokens", [1, 3, 64, 65, 128, 129, 1000])
def test_gradients_are_about_as_exact_as_their_type(torch, tokens, dtype):
    """In the 2-norm, against the exact gradients rounded once.  d in two parts, or in binary16 for bfloat16, adds at most 2^-3 of a rounding to each
    element, 2^-6 to its square; that of many binary16 tokens is rounded once itself, and adds another one: sqrt(2), and what the mantissas of a few
    hundred large elements do to it."""
    hidden, weight, ids, teacher = inputs(torch, tokens, 200, 3000, 24, dtype, seed=31, marked=0.1)
    hidden = (hidden.float() * 2).to(hidden.dtype)
    dloss = torch.full((tokens,), 1 / 3, device="cuda")
    got = call(torch, hidden, weight, ids, teacher, dloss)
    there, x, w = ids != -100, hidden.double(), weight.double()
    at = ids.clamp(min=0)
    q = torch.nan_to_num(torch.softmax(torch.where(there, teacher.double(), -math.inf), dim=1))
    d = torch.softmax(torch.mm(x, w.t()), dim=1).scatter_add_(1, at, -q) * dloss.double()[:, None] * there.any(dim=1)[:, None]
    most = 1.6 if dtype == "f16" and tokens > 128 else 1.05
    for got_, want in ((got["dhidden"], torch.mm(d, w)), (got["dweight"], torch.mm(d.t().contiguous(), x))):
        once = float((want.to(got_.dtype).double() - want).norm())
        assert float((got_.double() - want).norm()) <= most * once


@pytest.mark.parametrize("tokens", [100, 300])
@pytest.mark.parametrize("of_hidden, of_weight", [(2.0**30, 2.0**-30), (2.0**-40, 2.0**40), (2.0**-100, 1.0), (1.0, 2.0**-100), (2.0**9, 2.0**-9)])
def test_operands_of_any_size_in_bfloat16(torch, tokens, of_hidden, of_weight):
    """Powers of two change nothing but the results' own power where the logits stay what they are, and next to nothing where these vanish."""
    hidden, weight, ids, teacher = inputs(torch, tokens, 136, 900, 12, "bf16", seed=3)
    dloss = torch.full((tokens,), 0.5, device="cuda")
    check(torch, (hidden.float() * of_hidden).bfloat16(), (weight.float() * of_weight).bfloat16(), ids, teacher, dloss)
    weight.zero_()
    check(torch, hidden, weight, ids, teacher, dloss)


def test_operands_with_outliers_in_bfloat16(torch):
    hidden, weight, ids, teacher = inputs(torch, 300, 136, 900, 12, "bf16", seed=3)
    hidden[:, 7] *= 0.0
    hidden[11, 7] = 2.0**20
    weight[:, 7] *= 2.0**-20
    weight[5, 9] = 24.0
    check(torch, hidden, weight, ids, teacher, torch.full((300,), 0.5, device="cuda"))


@pytest.mark.parametrize("tokens", [40, 150])
def test_most_entries_in_a_few_columns(torch, tokens):
    """More than 63 in 64 columns: once, twice, at both ends of the vocabulary."""
    hidden, weight, ids, teacher = inputs(torch, tokens, 128, 20000, 1000, "bf16", seed=2, marked=0.0)
    ids[::3] = torch.arange(1000, device="cuda") % 100
    ids[1::3] = 19999 - torch.arange(1000, device="cuda") % 64
    ids[2::3, 100:163] = 320 + torch.arange(63, device="cuda")
    ids[5, 100:164] = 320 + torch.arange(64, device="cuda")
    ids[8] = 64
    check(torch, hidden, weight, ids, teacher, torch.full((tokens,), 0.1, device="cuda"))


@pytest.mark.parametrize("tokens", [3, 70, 140])
def test_the_widest_hidden_states(torch, tokens):
    check(torch, *inputs(torch, tokens, 1 << 17, 40, 8, "bf16", seed=1), torch.full((tokens,), 0.1, device="cuda"))


@pytest.mark.parametrize("tokens", [10, 150])
def test_an_entry_of_the_vocabulary_as_the_mark(torch, tokens):
    hidden, weight, ids, teacher = inputs(torch, tokens, 64, 50, 9, "f16", seed=1, marked=0.0)
    ids[4] = 7
    got = check(torch, hidden, weight, ids, teacher, torch.full((tokens,), 0.1, device="cuda"), ignore=7)
    assert got["loss"][4] == 0 and (got["dhidden"][4] == 0).all()


def test_two_calls_at_once_with_workspaces_of_their_own(torch):
    tokens, width, vocab, entries = 600, 256, 4000, 32
    args = [inputs(torch, tokens, width, vocab, entries, "bf16", seed=k) for k in range(2)]
    dloss = torch.full((tokens,), 0.01, device="cuda")
    alone = [call(torch, *a, dloss) for a in args]
    streams = [torch.cuda.Stream() for _ in range(2)]
    need = cgx.cgx_head_distill_workspace(tokens, width, vocab, entries, cgx.BF16, True)
    ws = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(2)]
    out = [{k: torch.empty_like(v) for k, v in a.items()} for a in alone]
    torch.cuda.synchronize()
    for _ in range(3):
        for a, o, w, s in zip(args, out, ws, streams):
            cgx.cgx_head_distill(*a, o["loss"], o["lse"], o["picked"], w, stream=s)
            cgx.cgx_head_distill_grad(*a, o["lse"], o["picked"], dloss, o["dhidden"], o["dweight"], w, stream=s)
    torch.cuda.synchronize()
    for a, o in zip(alone, out):
        assert all(torch.equal(a[k], o[k]) for k in a)
