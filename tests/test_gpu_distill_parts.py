"""d of few tokens is held in two parts of 16 bits, whose sum is d to some 2^-22: the second one has to be what the first one, as it is stored, leaves.

A hidden state has one element that is not 0, so that the weight's gradient is d times that, rounded once.  Tolerance, relative to
the probability p and to d: logits are exact here; lse is off by 1.2e-5 + 2^-23 |lse| at most and exp by 40 * 2^-23 (sums and
exponentials in binary32), the factor and its product by 2^-23, d by 2^-22 in two parts (half a subnormal step of the second one's,
2^-39 of the largest factor); and the result's own rounding, u of it, or half a subnormal step in binary16.
A first part that is off by a step of its own (2 u) and not made up for is outside.
"""
import math

import pytest

from test_gpu_distill import ROUNDOFF, call, dtype_of, torch  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("vocab", [2000, 5000, 50257])          # (up to 64 tiles of logits, and more)
@pytest.mark.parametrize("tokens", [64, 128])
def test_the_parts_are_of_one_number(torch, tokens, vocab, dtype):
    g = torch.Generator().manual_seed(vocab)
    dt = dtype_of(torch, dtype)
    each = torch.tensor([1.25, 1.5, 1.75])[torch.arange(tokens) % 3]
    hidden = torch.diag(each).to(dt).cuda()
    weight = (torch.randn(vocab, tokens, generator=g) * 2).to(dt).cuda()
    ids = torch.randint(0, vocab, (tokens, 1), generator=g).cuda()
    dloss = (torch.logspace(-1, 0, tokens) * 1024).cuda()
    got = call(torch, hidden, weight, ids, torch.zeros(tokens, 1, device="cuda"), dloss)["dweight"].double().t()
    each = each.double().cuda()[:, None]
    z = weight.double().t() * each
    lse = torch.logsumexp(z, dim=1, keepdim=True)
    p = torch.exp(z - lse)
    factor = dloss.double()[:, None]
    d = factor * p.scatter_add(1, ids, -torch.ones(tokens, 1, dtype=torch.float64, device="cuda"))
    bound = factor * p * (1.2e-5 + 2.0**-23 * lse.abs() + 40 * 2.0**-23) + 2.0**-21 * d.abs() + 1024 * 2.0**-39
    d, bound = d * each, bound * each * 1.01
    bound = bound + ROUNDOFF[dtype] * (d.abs() + bound) + (2.0**-25 if dtype == "f16" else 0.0)
    worst = float(((got - d).abs() / bound).max())
    assert worst <= 1.0 and not math.isnan(worst)
