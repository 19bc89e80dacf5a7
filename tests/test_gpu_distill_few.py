"""Distillation of up to 128 tokens, which has kernels of its own for the gradients, beside more of them: what tokens that take no part hold changes nothing for
the others, whatever it is, and whichever kernels form d."""
import pytest

from test_gpu_distill import TYPES, call, check, inputs, torch  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu

TOKENS = [12, 40, 100, 128, 129, 200]
VOCABS = [700, 5000]                                            # up to 64 tiles of 64 x 64 logits for all of these numbers of tokens but 200, and more


def without_part(torch, ids, teacher, off):
    """Every second of these tokens gets no entry at all, the others entries of no share."""
    n = torch.arange(len(off), device="cuda")
    ids, teacher = ids.clone(), teacher.clone()
    ids[off] = -100
    teacher[off] = float("nan")
    half = off & (n % 2 == 0)
    ids[half] = 3
    teacher[half] = float("-inf")
    return ids, teacher


@pytest.mark.parametrize("large", [2.0**20, 1e9, 3e38, float("inf"), float("nan")])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("tokens", TOKENS)
def test_a_factor_of_a_token_that_takes_no_part_changes_nothing(torch, tokens, vocab, dtype, large):
    """d is held in units of the largest factor of those that do."""
    hidden, weight, ids, teacher = inputs(torch, tokens, 72, vocab, 20, dtype, seed=tokens, marked=0.0)
    off = torch.arange(tokens, device="cuda") % 3 == 1
    ids, teacher = without_part(torch, ids, teacher, off)
    dloss = torch.linspace(0.001, 0.002, tokens, device="cuda")
    dloss[5] *= -1
    want = check(torch, hidden, weight, ids, teacher, torch.where(off, 0.0, dloss))
    got = call(torch, hidden, weight, ids, teacher, torch.where(off, large, dloss))
    assert all(torch.equal(got[k], want[k]) for k in want)


@pytest.mark.parametrize("entries", [1, 7, 8, 9, 65, 300])
@pytest.mark.parametrize("first", [True, False])
def test_the_only_entry_of_the_token_with_the_largest_factor(torch, entries, first):
    """It may be anywhere in its row.  An id outside the vocabulary makes a token take part too: the others' rows are what they are beside one inside."""
    tokens, at = 70, 0 if first else entries - 1
    hidden, weight, ids, teacher = inputs(torch, tokens, 64, 900, entries, "f16", seed=3, marked=0.0)
    ids[66] = -100
    ids[66, at] = 17
    dloss = torch.full((tokens,), 2.5e-4, device="cuda")
    dloss[66] = 1e3
    want = check(torch, hidden, weight, ids, teacher, dloss)
    ids[66, at] = 900
    got = call(torch, hidden, weight, ids, teacher, dloss)
    others = torch.arange(tokens, device="cuda") != 66
    assert got["dhidden"][66].isnan().all() and torch.equal(got["dhidden"][others], want["dhidden"][others])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("tokens", TOKENS)
def test_a_hidden_state_of_a_token_that_takes_no_part_changes_nothing(torch, tokens, vocab, dtype):
    width = 136
    hidden, weight, ids, teacher = inputs(torch, tokens, width, vocab, 6, dtype, seed=9, marked=0.0)
    n = torch.arange(tokens, device="cuda")
    dloss = torch.full((tokens,), 0.5, device="cuda")
    for off in (n % 3 == 1, n < tokens - 2, n > 1, n >= 0, n != tokens // 2):
        at, logits = without_part(torch, ids, teacher, off)
        x = hidden.clone()
        x[off] = 0.0
        want = check(torch, x, weight, at, logits, dloss)
        x[off] = torch.tensor([float("nan"), float("inf")], dtype=hidden.dtype, device="cuda").repeat(width // 2)
        got = call(torch, x, weight, at, logits, dloss)
        assert all(torch.equal(got[k], want[k]) for k in want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("tokens", TOKENS)
def test_a_factor_of_zero_takes_no_part_in_the_gradients(torch, tokens, vocab, dtype):
    """Its hidden state may hold anything, its loss is what it is."""
    width = 72
    hidden, weight, ids, teacher = inputs(torch, tokens, width, vocab, 6, dtype, seed=10, marked=0.0)
    off = torch.arange(tokens, device="cuda") % 4 == 2
    dloss = torch.where(off, 0.0, 0.5)
    want = check(torch, hidden, weight, ids, teacher, dloss)
    hidden[off] = torch.tensor([float("nan"), float("inf")], dtype=hidden.dtype, device="cuda").repeat(width // 2)
    got = call(torch, hidden, weight, ids, teacher, dloss)
    assert all(torch.equal(got[k], want[k]) for k in ("dhidden", "dweight"))
    assert got["loss"][off].isnan().all() and torch.equal(got["loss"][~off], want["loss"][~off])


@pytest.mark.parametrize("scale", [2.0**-20, 1.0, 4096.0])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("tokens", TOKENS)
def test_uneven_factors(torch, tokens, vocab, dtype, scale):
    hidden, weight, ids, teacher = inputs(torch, tokens, 128, vocab, 50, dtype, seed=8)
    dloss = scale * torch.logspace(-3, 0, tokens, device="cuda") / 64
    dloss[::5] *= -1
    check(torch, hidden, weight * 0.125 if scale > 1 else weight, ids, teacher, dloss, temperature=2.0)
