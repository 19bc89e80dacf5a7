"""A distillation step of a student with a tied table, run as a program runs it: lookup, loss and gradients from a teacher's entries, the lookup's gradient
added to the head's, norm, clipping and fusing, compression.  Against the formulas in 64 bits."""
import math

import numpy as np
import pytest

from paper_2111_08617_amd import binding as cgx

pytestmark = pytest.mark.gpu

TOKENS, WIDTH, VOCAB, ENTRIES, TEMPERATURE, IGNORE = 700, 192, 3001, 12, 2.0, -100
SCALE = math.sqrt(WIDTH)


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available(), "these tests need the MI355X"
    cgx.lib()
    return t


class Step:
    """Everything that a program keeps, and its step; `dt` of the table."""

    def __init__(self, torch, dtype):
        self.torch = torch
        dt = {torch.float32: cgx.F32, torch.bfloat16: cgx.BF16, torch.float16: cgx.F16}[dtype]
        g = torch.Generator().manual_seed(3)
        self.table = (torch.randn(VOCAB, WIDTH, generator=g) / SCALE).to(dtype).cuda()
        self.hidden, self.dhidden = (torch.empty(TOKENS, WIDTH, dtype=dtype, device="cuda") for _ in range(2))
        self.dtable = torch.empty_like(self.table)
        self.loss, self.lse = torch.empty(2, TOKENS, device="cuda")
        self.picked = torch.empty(TOKENS, ENTRIES, device="cuda")
        self.tokens, self.ids = torch.zeros(TOKENS, dtype=torch.int64, device="cuda"), torch.zeros(TOKENS, ENTRIES, dtype=torch.int64, device="cuda")
        self.teacher, self.dloss = torch.zeros(TOKENS, ENTRIES, device="cuda").half(), torch.zeros(TOKENS, device="cuda")
        self.head_workspace = torch.empty(cgx.cgx_head_distill_workspace(TOKENS, WIDTH, VOCAB, ENTRIES, dt, True), dtype=torch.uint8, device="cuda")
        self.embed_workspace = torch.empty(cgx.cgx_embed_grad_workspace(TOKENS, WIDTH, VOCAB, dt), dtype=torch.uint8, device="cuda")
        self.norm_workspace = torch.empty(cgx.cgx_grad_norm_workspace(), dtype=torch.uint8, device="cuda")
        self.norm = torch.empty(1, device="cuda")
        self.plan = cgx.Plan(np.array([0, VOCAB * WIDTH]), np.array([8], np.uint8), bucket=128, dt=cgx.F32)
        packed, meta = cgx.cgx_sizes(self.plan)
        self.fused = torch.empty(self.plan.n, device="cuda")
        self.packed, self.meta = torch.empty(packed, dtype=torch.uint8, device="cuda"), torch.empty(meta // 4, device="cuda")
        cgx.cgx_quantize(self.fused.zero_(), self.plan, 1, self.packed, self.meta)       # (the plan's table, ahead of any capture)

    def batch(self, seed):
        torch, g = self.torch, self.torch.Generator().manual_seed(seed)
        self.tokens.copy_((torch.rand(TOKENS, generator=g) ** 3 * VOCAB).long())
        self.tokens[::9] = IGNORE
        self.ids.copy_(torch.randint(0, VOCAB, (TOKENS, ENTRIES), generator=g))
        self.ids[::9] = IGNORE
        self.teacher.copy_(torch.randn(TOKENS, ENTRIES, generator=g) * 2)
        self.dloss.copy_(torch.where(self.tokens == IGNORE, 0.0, TEMPERATURE ** 2 / TOKENS))

    def __call__(self):
        cgx.cgx_embed(self.table, self.tokens, self.hidden, scale=SCALE, ignore=IGNORE)
        cgx.cgx_head_distill(self.hidden, self.table, self.ids, self.teacher, self.loss, self.lse, self.picked, self.head_workspace,
                             temperature=TEMPERATURE, ignore=IGNORE)
        cgx.cgx_head_distill_grad(self.hidden, self.table, self.ids, self.teacher, self.lse, self.picked, self.dloss, self.dhidden, self.dtable,
                                  self.head_workspace, temperature=TEMPERATURE, ignore=IGNORE)
        cgx.cgx_embed_grad(self.dhidden, self.tokens, self.dtable, self.embed_workspace, scale=SCALE, ignore=IGNORE, accumulate=True)
        cgx.cgx_grad_norm([self.dtable], self.norm, self.norm_workspace)
        cgx.cgx_grad_clip([self.dtable], self.norm, 0.05, out=self.fused)
        cgx.cgx_quantize(self.fused, self.plan, 7, self.packed, self.meta)

    def want(self):
        """(losses, gradient of the tied table) in 64 bits."""
        torch = self.torch
        table = self.table.cpu().double().requires_grad_()
        rows = torch.nonzero(self.tokens.cpu() != IGNORE)[:, 0]
        ids = self.ids.cpu()[rows]
        hidden = table[self.tokens.cpu()[rows]] * float(np.float32(SCALE))
        logp = torch.log_softmax(hidden @ table.t() / TEMPERATURE, dim=1).gather(1, ids)
        q = torch.softmax(self.teacher.cpu()[rows].double() / TEMPERATURE, dim=1)
        loss = (q * (q.log() - logp)).sum(dim=1)
        (loss * self.dloss.cpu()[rows].double()).sum().backward()
        return rows, loss.detach(), table.grad


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_a_step(torch, dtype):
    """Relative 2-norms: the hidden states, d (or its upper part), dhidden, the head's dtable and the sum of both gradients are rounded once each, by at most u
    of what they hold; a hidden state's rounding changes logits of size |z| by u |z| and probabilities with them (|z| up to some 5 here); the parts' norms are
    at most a few times the sum's."""
    step = Step(torch, getattr(torch, dtype))
    u = {"float32": 2.0**-24, "bfloat16": 2.0**-8, "float16": 2.0**-11}[dtype]
    for seed in (1, 2):
        step.batch(seed)
        step()
        rows, loss, grad = step.want()
        assert (step.loss[step.tokens == IGNORE] == 0).all()
        assert float((step.loss.cpu().double()[rows] - loss).norm() / loss.norm()) <= 10 * u + 1e-5
        got = step.dtable.cpu().double()
        assert float((got - grad).norm() / grad.norm()) <= 20 * u + 1e-5
        norm = float(got.norm())
        assert abs(float(step.norm) - norm) <= 2.0**-22 * norm
        assert torch.allclose(step.fused.cpu().double().view_as(got), got * min(1.0, 0.05 / norm), rtol=1e-6, atol=0)
        out = torch.empty_like(step.fused)
        cgx.cgx_dequantize(step.packed, step.meta, step.plan, cgx.F32, out)
        assert float((out - step.fused).abs().max()) <= float(step.fused.max() - step.fused.min()) / 255 * 1.01


def test_a_captured_step(torch):
    step = Step(torch, torch.bfloat16)
    step.batch(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (5, 6, 7):
        step.batch(seed)
        for ws in (step.head_workspace, step.embed_workspace):
            ws.fill_(0xff)
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in (step.hidden, step.loss, step.lse, step.picked, step.dhidden, step.dtable, step.norm, step.fused, step.packed, step.meta)]
        step()
        torch.cuda.synchronize()
        now = (step.hidden, step.loss, step.lse, step.picked, step.dhidden, step.dtable, step.norm, step.fused, step.packed, step.meta)
        assert all(torch.equal(a, b) for a, b in zip(replayed, now))
