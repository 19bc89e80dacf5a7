"""cgx_grad_norm and cgx_grad_clip on the GPU against sums in 64 bits.

The norm is summed in binary64 and rounded once: within 2^-23 of the exact one, relative (2^-24 of the rounding, the rest far
below).  A clipped element is one binary32 product of the element and max_norm / norm, rounded once more to the type it is stored in:
given the norm that the call used, the same bits as torch's binary32 arithmetic on the host gives.
"""
import math

import numpy as np
import pytest

from paper_2111_08617_amd import binding as cgx
from paper_2111_08617_amd import workloads as wl

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available(), "these tests need the MI355X"
    cgx.lib()
    return t


def tensors(torch, sizes, kinds, seed=0, odd=True, scale=1.0):
    """Gradients of the sizes, types in turn, each starting at an element of its own of a larger buffer."""
    types = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
    g = torch.Generator().manual_seed(seed)
    out = []
    for k, n in enumerate(sizes):
        start = (k * 3 + 1) % 8 if odd else 0
        buf = torch.full((n + 16,), 11.0, dtype=types[kinds[k % len(kinds)]], device="cuda")
        part = buf[start:start + n]
        part.copy_(torch.randn(n, generator=g) * scale * 10.0 ** (k % 4 - 2))
        out.append(part)
    return out


def norm_of(torch, grads, stream=None):
    ws = torch.full((cgx.cgx_grad_norm_workspace(),), 0xff, dtype=torch.uint8, device="cuda")
    norm = torch.full((3,), -1.0, device="cuda")
    cgx.cgx_grad_norm(grads, norm[1:2], ws, stream=stream)
    torch.cuda.synchronize()
    assert norm[0] == -1.0 and norm[2] == -1.0
    return norm[1:2]


def exact(grads):
    return math.sqrt(math.fsum(float(np.sum(g.cpu().double().numpy() ** 2)) for g in grads))


SIZES = {
    "one": [1], "none": [], "empty": [0, 0], "short": [1, 2, 7, 8, 9, 0, 15, 16, 17, 63, 64, 65],
    "items": [8191, 8192, 8193, 0, 16384, 16385, 24575, 0],
    "many": [(k * 37) % 300 for k in range(500)],
    "full groups": [5] * 160 + [0] * 40 + [3] * 160,
    "long": [3000001, 5, 40960, 1 << 20],
}
KINDS = [("f32",), ("f16",), ("bf16",), ("f32", "bf16", "f16")]


@pytest.mark.parametrize("kinds", KINDS, ids="-".join)
@pytest.mark.parametrize("sizes", SIZES)
def test_norm(torch, sizes, kinds):
    grads = tensors(torch, SIZES[sizes], kinds, seed=len(sizes))
    got, want = float(norm_of(torch, grads)), exact(grads)
    assert abs(got - want) <= 2.0**-23 * want
    assert torch.equal(norm_of(torch, grads), norm_of(torch, grads)), "not the same bits again"


def test_more_elements_than_all_blocks_take_at_once(torch):
    sizes = [2048 * 8192 + 5, 3, 8192 * 700 + 1]
    grads = tensors(torch, sizes, ("bf16", "f32"), odd=True)
    got, want = float(norm_of(torch, grads)), exact(grads)
    assert abs(got - want) <= 2.0**-23 * want


def test_norms_outside_what_binary32_squares_hold(torch):
    for size in (1e30, 1e-30, 1e-42):
        grads = [torch.full((1000,), size, device="cuda"), torch.zeros(5, device="cuda")]
        got, want = float(norm_of(torch, grads)), exact(grads)
        assert abs(got - want) <= 2.0**-23 * want + 2.0**-149
    assert math.isinf(float(norm_of(torch, [torch.full((100,), 3e38, device="cuda")])))
    assert float(norm_of(torch, [torch.zeros(100, device="cuda")])) == 0.0


def test_nan_and_infinity_reach_the_norm_and_the_clipped_tensors(torch):
    grads = tensors(torch, [100, 9000], ("f32",))
    grads[1][8500] = float("inf")
    norm = norm_of(torch, grads)
    assert math.isinf(float(norm))
    out = torch.full((9100,), 5.0, device="cuda")
    cgx.cgx_grad_clip(grads, norm, 1.0, out=out)
    assert int(out.isnan().sum()) == 1 and int((out == 0).sum()) == 9099
    grads[0][3] = float("nan")
    norm = norm_of(torch, grads)
    assert math.isnan(float(norm))
    cgx.cgx_grad_clip(grads, norm, 1.0, out=out)
    assert out.isnan().all()


def expected(torch, grads, norm, max_norm, dtype=None):
    norm = norm.cpu()
    factor = torch.tensor([max_norm], dtype=torch.float32) / norm if float(norm) > max_norm else torch.ones(1)
    return [(g.cpu().float() * factor).to(dtype or g.dtype) for g in grads]


def same_bits(torch, a, b):
    kind = torch.int32 if a.dtype == torch.float32 else torch.int16
    return torch.equal(a.cpu().view(kind), b.cpu().view(kind))


@pytest.mark.parametrize("kinds", KINDS, ids="-".join)
@pytest.mark.parametrize("sizes", SIZES)
def test_clip_in_place(torch, sizes, kinds):
    grads = tensors(torch, SIZES[sizes], kinds, seed=3)
    total = exact(grads)
    norm = norm_of(torch, grads)
    max_norm = float(np.float32(total / 3))
    want = expected(torch, grads, norm, max_norm)
    cgx.cgx_grad_clip(grads, norm, max_norm)
    torch.cuda.synchronize()
    for g, w in zip(grads, want):
        assert same_bits(torch, g, w)
        around = torch.cat([g.as_strided((g.storage_offset(),), (1,), 0), g.as_strided((16 - g.storage_offset(),), (1,), g.storage_offset() + g.numel())])
        assert (around == 11.0).all(), "wrote beside a tensor"


@pytest.mark.parametrize("out", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("kinds", KINDS, ids="-".join)
@pytest.mark.parametrize("sizes", SIZES)
def test_clip_into_the_fused_buffer(torch, sizes, kinds, out):
    grads = tensors(torch, SIZES[sizes], kinds, seed=4)
    dtype = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[out]
    norm = norm_of(torch, grads)
    before = [g.clone() for g in grads]
    n = sum(SIZES[sizes])
    fused = torch.full((n + 64,), -7.0, dtype=dtype, device="cuda")
    for share in (0.25, 4.0):                                   # clipped, and left as they are
        max_norm = float(np.float32(exact(grads) * share))
        cgx.cgx_grad_clip(grads, norm, max_norm, out=fused)
        torch.cuda.synchronize()
        want = torch.cat(expected(torch, grads, norm, max_norm, dtype) or [torch.zeros(0, dtype=dtype)])
        assert same_bits(torch, fused[:n], want) and (fused[n:] == -7.0).all()
    for g, b in zip(grads, before):
        assert torch.equal(g, b)


def test_a_norm_under_the_limit_leaves_the_tensors_alone(torch):
    grads = tensors(torch, [5000, 20000], ("f16", "f32"), seed=5)
    grads[0][17] = -0.0
    before = [g.clone() for g in grads]
    cgx.cgx_grad_clip(grads, norm_of(torch, grads), 1e9)
    for g, b in zip(grads, before):
        assert same_bits(torch, g, b)


def test_the_clipped_buffer_is_what_the_quantizer_takes(torch, oracle):
    """Mixed gradients of a plan's layers, clipped into its fused buffer and quantized: the oracle's bytes for that buffer."""
    w = wl.tiny_mixed(seed=11, bucket=128)
    sizes = [int(s) for s in np.diff(w.offsets)]
    grads = tensors(torch, sizes, ("f32", "bf16", "f16"), seed=6)
    plan = cgx.Plan(w.offsets, w.bits, w.bucket, w.dt)
    fused = torch.empty(plan.n, device="cuda")
    cgx.cgx_grad_clip(grads, norm_of(torch, grads), 0.5, out=fused)
    pb, mb = cgx.cgx_sizes(plan)
    packed, meta = torch.empty(pb, dtype=torch.uint8, device="cuda"), torch.empty(mb // 4, device="cuda")
    cgx.cgx_quantize(fused, plan, 5, packed, meta)
    torch.cuda.synchronize()
    assert abs(float(fused.double().norm()) - 0.5) < 2e-3 * 0.5          # elements of 16-bit tensors are exact, the products rounded
    p, m = oracle.quantize(fused.cpu().numpy(), w.offsets, w.bits, w.bucket, 5, w.dt)
    assert np.array_equal(packed.cpu().numpy(), p) and meta.cpu().numpy().tobytes() == m.tobytes()


def test_streams_and_graphs(torch):
    grads = tensors(torch, [(k * 911) % 20000 for k in range(200)], ("f32", "f16"), seed=7)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    assert torch.equal(norm_of(torch, grads), norm_of(torch, grads, stream=side))
    ws = torch.empty(cgx.cgx_grad_norm_workspace(), dtype=torch.uint8, device="cuda")
    norm, fused = torch.empty(1, device="cuda"), torch.empty(sum(g.numel() for g in grads), device="cuda")

    def step():
        cgx.cgx_grad_norm(grads, norm, ws)
        cgx.cgx_grad_clip(grads, norm, 2.0, out=fused)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        for g in grads:
            g.mul_(1.0 + k)
        step()
        torch.cuda.synchronize()
        want = norm.clone(), fused.clone()
        norm.fill_(0.0)
        fused.fill_(0.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(norm, want[0]) and torch.equal(fused, want[1])


@pytest.mark.parametrize("odd", [False, True])
def test_lengths_around_an_items_and_lists_around_a_launchs(torch, odd):
    """Items of 4096 elements, 240 tensors a launch, results above and below the size from which they are streamed."""
    for sizes in ([4095, 4096, 4097, 0, 8191, 1], [3] * 239, [3] * 240, [3] * 241, [2] * 480 + [0] * 5 + [7], [1 << 25, 4097, 3 << 22]):
        grads = tensors(torch, sizes, ("bf16", "f32", "f16"), seed=len(sizes), odd=odd)
        norm, total = norm_of(torch, grads), exact(grads)
        assert abs(float(norm) - total) <= 2.0**-23 * total
        max_norm = float(np.float32(total / 2))
        want = torch.cat(expected(torch, grads, norm, max_norm, torch.float32))
        fused = torch.full((sum(sizes) + 64,), -7.0, device="cuda")
        cgx.cgx_grad_clip(grads, norm, max_norm, out=fused)
        torch.cuda.synchronize()
        assert same_bits(torch, fused[:sum(sizes)], want) and (fused[sum(sizes):] == -7.0).all()
        in_place = expected(torch, grads, norm, max_norm)
        cgx.cgx_grad_clip(grads, norm, max_norm)
        torch.cuda.synchronize()
        assert all(same_bits(torch, g, w) for g, w in zip(grads, in_place))


def test_lists_beyond_the_memory_side_cache(torch):
    """More than 256 MB of gradients of three types, each starting at an odd element: the norm's loads and the clipping's stores past the
    caches, in place and into a fused buffer of each type (230 MB and more).  The results are formed on the device, by the same binary32
    arithmetic that torch's elementwise operations are."""
    sizes = [(33 << 20) + 5, (49 << 20) + 1, (37 << 20) + 3, 4097, 0, 7]
    kinds = ("f32", "bf16", "f16")

    def fresh():
        g = torch.Generator(device="cuda").manual_seed(31)
        out = []
        for k, n in enumerate(sizes):
            buf = torch.full((n + 16,), 11.0, dtype={"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[kinds[k % 3]], device="cuda")
            part = buf[2 * k + 1:2 * k + 1 + n]
            part.copy_(torch.randn(n, generator=g, device="cuda") * 10.0 ** -(k % 3))
            out.append(part)
        return out

    def bits(t):
        return t.view(torch.int32 if t.dtype == torch.float32 else torch.int16)

    grads = fresh()
    assert sum(g.numel() * g.element_size() for g in grads) > 256 << 20
    want = math.sqrt(math.fsum(float(part.double().square().sum()) for g in grads for part in g.split(1 << 24)))
    norm = norm_of(torch, grads)
    assert abs(float(norm) - want) <= 2.0**-23 * want
    assert torch.equal(norm, norm_of(torch, grads)), "not the same bits again"
    max_norm = float(np.float32(want / 3))
    factor = (torch.tensor([max_norm], dtype=torch.float32) / norm.cpu()).cuda()
    total = sum(sizes)
    for dtype in (torch.float32, torch.float16, torch.bfloat16):
        fused = torch.full((total + 64,), -7.0, dtype=dtype, device="cuda")
        assert total * fused.element_size() > 128 << 20
        cgx.cgx_grad_clip(grads, norm, max_norm, out=fused)
        at = 0
        for g in grads:
            assert torch.equal(bits(fused[at:at + g.numel()]), bits((g.float() * factor).to(dtype)))
            at += g.numel()
        assert (fused[total:] == -7.0).all()
    cgx.cgx_grad_clip(grads, norm, max_norm)
    for g, before in zip(grads, fresh()):
        assert torch.equal(bits(g), bits((before.float() * factor).to(before.dtype)))
        around = torch.cat([g.as_strided((g.storage_offset(),), (1,), 0), g.as_strided((16 - g.storage_offset(),), (1,), g.storage_offset() + g.numel())])
        assert (around == 11.0).all(), "wrote beside a tensor"


@pytest.mark.parametrize("out", ["f32", "f16", "bf16"])
def test_an_infinite_limit_converts_and_fuses(torch, out):
    grads = tensors(torch, [5000, 0, 4097, 33], ("f32", "bf16", "f16"), seed=8)
    dtype = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[out]
    for norm in (0.0, 3.0, math.inf):
        fused = torch.full((9130 + 64,), -7.0, dtype=dtype, device="cuda")
        cgx.cgx_grad_clip(grads, torch.tensor([norm], device="cuda"), math.inf, out=fused)
        assert same_bits(torch, fused[:9130], torch.cat([g.to(dtype) for g in grads])) and (fused[9130:] == -7.0).all()
    cgx.cgx_grad_clip(grads, torch.tensor([math.nan], device="cuda"), math.inf, out=fused)
    assert fused[:9130].isnan().all()
