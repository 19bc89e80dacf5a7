"""A teacher's logits count by their differences: what all of a token's have in common changes nothing, however large it is.

Tolerances.  With s the logits over a temperature that is a power of two (exact), top their largest, t = s - top (one rounding, 2^-24 |t|):
  q: exp of t (2^-23 and t's error), a sum of at most 1024 terms in 64 lanes (22 * 2^-24), a division: relative 2^-23 (2 + |t|) + 22 * 2^-24
  log q = t - log(sum): t's error, the logarithm's (2^-22 of 1 + its size, its argument's 22 * 2^-24), the difference's 2^-24 of both
  loss = sum q (log q + (lse - picked / T)): errors of lse and of picked as in the other tests, 2^-23 of both for each difference and sum, sums of the terms.
"""
import math

import pytest

from test_gpu_distill import TYPES, call, inputs, torch  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


def check_loss(torch, hidden, weight, ids, teacher, temperature):
    got = call(torch, hidden, weight, ids, teacher, temperature=temperature)
    width, entries, t = hidden.shape[1], ids.shape[1], temperature
    there = ids != -100
    assert there.any(dim=1).all()
    at = torch.where(there, ids, 0)
    x, w = hidden.double(), weight.double()
    z = torch.mm(x, w.t())
    off_z = (width + 2) * 2.0**-24 * torch.mm(x.abs(), w.abs().t()) / t + 2.0**-23 * z.abs() / t
    lse = torch.logsumexp(z / t, dim=1, keepdim=True)
    off_lse = off_z.max(dim=1, keepdim=True).values + 1.2e-5 + 2.0**-23 * lse.abs()
    picked, off_picked = z.gather(1, at) / t, off_z.gather(1, at)
    soft = torch.where(there, teacher.double(), -math.inf) / t
    soft = soft - soft.max(dim=1, keepdim=True).values
    mass = torch.logsumexp(soft, dim=1, keepdim=True)
    q = torch.exp(soft - mass)
    size = torch.where(q > 0, soft.abs(), 0.0)
    term = torch.where(q > 0, torch.where(q > 0, soft, 0.0) - mass + lse - picked, 0.0)
    off_q = 2.0**-23 * (2 + size) + 22 * 2.0**-24
    off = off_q * term.abs() + off_lse + off_picked + 2.0**-23 * size + 2.0**-22 * (1 + mass.abs()) + 22 * 2.0**-24
    off = q * (off + 2.0**-23 * (size + mass + lse.abs() + picked.abs() + term.abs()) + entries * 2.0**-24 * term.abs())
    loss = (q * term).sum(dim=1)
    assert ((got["loss"].double() - loss).abs() <= off.sum(dim=1) + 2.0**-23 * loss.abs()).all()
    return got


@pytest.mark.parametrize("temperature", [2.0**-10, 0.5, 1.0, 4.0])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens", [1, 12, 40, 200])
def test_a_common_offset_changes_nothing(torch, tokens, dtype, temperature):
    """Logits in steps of 2^-6 up to 8, so that sums with any of these offsets are exact in binary32."""
    hidden, weight, ids, _ = inputs(torch, tokens, 72, 900, 20, dtype, seed=tokens)
    ids[:, 3] = 5
    g = torch.Generator().manual_seed(1)
    teacher = (torch.randint(0, 512, (tokens, 20), generator=g) / 64).cuda() * min(temperature, 1.0)
    want = check_loss(torch, hidden, weight, ids, teacher, temperature)
    for offset in (4096.0, -(2.0**14), 2.0**16):
        got = check_loss(torch, hidden, weight, ids, teacher + offset * min(temperature, 1.0), temperature)
        assert all(torch.equal(got[k], want[k]) for k in want)


@pytest.mark.parametrize("tokens", [5, 70])
def test_low_temperatures_and_large_logits(torch, tokens):
    hidden, weight, ids, teacher = inputs(torch, tokens, 72, 900, 20, "f32", seed=tokens)
    ids[:, 3] = 5
    check_loss(torch, hidden, weight, ids, teacher + 9.0, 2.0**-10)
    check_loss(torch, hidden, weight, ids, teacher * 1e-2 + 3e4, 1.0)
