"""Host-side tests of the head's and the gradients' calls: sizes, refusals, the binding's checks.  No kernel is launched."""
import ctypes
import os

import numpy as np
import pytest

from paper_2111_08617_amd import binding as cgx

P, ODD = 0x10000, 0x10001          # addresses that pass and fail the alignment checks; nothing is read before a refusal


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(cgx.LIB_PATH):
        from paper_2111_08617_amd import build
        build.build()
    return cgx.lib()


OK, NULL, SIZE, DTYPE, ALIGN = 0, -1, -2, -7, -9


def test_workspace_grows_with_the_tokens_and_not_with_the_logits(lib):
    sizes = [cgx.cgx_head_workspace(n, 2048, 50257, cgx.BF16, True) for n in (1, 100, 1024, 8192, 65536)]
    assert sizes == sorted(sizes)
    # far below the logits' size in binary32, at every length
    assert sizes[-1] < 65536 * 50257 * 4 / 4
    forward = cgx.cgx_head_workspace(8192, 2048, 50257, cgx.BF16)
    assert forward < 8192 * 50257 * 2 / 4
    for dt in (cgx.F32, cgx.F16, cgx.BF16):
        for n, h, v in ((0, 1, 1), (1, 1, 1), (3, 7, 11), (4096, 768, 30522)):
            assert 0 < cgx.cgx_head_workspace(n, h, v, dt) <= cgx.cgx_head_workspace(n, h, v, dt, True)


@pytest.mark.parametrize("tokens, width, vocab, dt, want", [
    (-1, 64, 100, 0, SIZE), (1 << 24, 64, 100, 0, SIZE), (1, 0, 100, 0, SIZE), (1, -5, 100, 0, SIZE), (1, (1 << 17) + 1, 100, 0, SIZE),
    (1, 64, 0, 0, SIZE), (1, 64, 1 << 31, 0, SIZE), (1, 64, 100, 3, DTYPE), (1, 64, 100, -1, DTYPE)])
def test_head_sizes_that_are_refused(lib, tokens, width, vocab, dt, want):
    n = ctypes.c_size_t()
    assert lib.cgx_head_workspace(tokens, width, vocab, dt, 1, ctypes.byref(n)) == want
    assert lib.cgx_head_loss(P, P, P, tokens, width, vocab, dt, -100, P, P, P, 1 << 60, None) == want
    assert lib.cgx_head_loss_grad(P, P, P, P, P, tokens, width, vocab, dt, -100, P, P, P, 1 << 60, None) == want


def test_head_pointers_that_are_refused(lib):
    n = ctypes.c_size_t()
    assert lib.cgx_head_workspace(4, 64, 100, 0, 1, None) == NULL
    assert lib.cgx_head_workspace(4, 64, 100, 0, 1, ctypes.byref(n)) == OK
    # hidden, weight, targets | loss, lse, workspace
    for k in range(6):
        args = [P] * 6
        args[k] = None
        assert lib.cgx_head_loss(*args[:3], 4, 64, 100, 0, -100, *args[3:], 1 << 60, None) == NULL
        args[k] = ODD
        assert lib.cgx_head_loss(*args[:3], 4, 64, 100, 0, -100, *args[3:], 1 << 60, None) == ALIGN
    # hidden, weight, targets, lse, dloss | dhidden, dweight, workspace
    for k in range(8):
        args = [P] * 8
        args[k] = None
        assert lib.cgx_head_loss_grad(*args[:5], 4, 64, 100, 0, -100, *args[5:], 1 << 60, None) == NULL
        args[k] = ODD
        assert lib.cgx_head_loss_grad(*args[:5], 4, 64, 100, 0, -100, *args[5:], 1 << 60, None) == ALIGN
    assert lib.cgx_head_loss_grad(*[P] * 5, 4, 64, 100, 0, -100, P, P, P, n.value - 1, None) == SIZE
    forward = ctypes.c_size_t()
    assert lib.cgx_head_workspace(4, 64, 100, 0, 0, ctypes.byref(forward)) == OK
    assert lib.cgx_head_loss(P, P, P, 4, 64, 100, 0, -100, P, P, P, forward.value - 1, None) == SIZE
    # no tokens: nothing to do, nothing needed
    assert lib.cgx_head_loss(None, None, None, 0, 64, 100, 0, -100, None, None, None, 0, None) == OK
    assert lib.cgx_head_loss_grad(None, None, None, None, None, 0, 64, 100, 0, -100, None, None, None, 0, None) == NULL


def entries(*items):
    return (cgx._Tensor * max(len(items), 1))(*[cgx._Tensor(*i) for i in items])


@pytest.mark.parametrize("items, want", [
    ([(P, -1, 0, 0)], SIZE), ([(P, 1 << 43, 0, 0)], SIZE), ([(P, 4, 3, 0)], DTYPE), ([(P, 4, -1, 0)], DTYPE), ([(None, 4, 0, 0)], NULL),
    ([(P, 4, 0, 0), (P + 2, 4, 0, 0)], ALIGN), ([(P + 1, 4, 1, 0)], ALIGN), ([(P, 4, 0, 0), (P + 1, 4, 2, 0)], ALIGN)])
def test_gradient_lists_that_are_refused(lib, items, want):
    e = entries(*items)
    assert lib.cgx_grad_norm(e, len(items), P, P, 1 << 30, None) == want
    assert lib.cgx_grad_clip(e, len(items), P, 1.0, None, 0, None) == want
    assert lib.cgx_grad_clip(e, len(items), P, 1.0, P, 0, None) == want


def test_gradient_arguments_that_are_refused(lib):
    need = cgx.cgx_grad_norm_workspace()
    assert need > 0 and lib.cgx_grad_norm_workspace(None) == NULL
    e = entries((P, 4, 0, 0))
    assert lib.cgx_grad_norm(None, 1, P, P, need, None) == NULL
    assert lib.cgx_grad_norm(e, -1, P, P, need, None) == SIZE
    assert lib.cgx_grad_norm(e, 1, None, P, need, None) == NULL
    assert lib.cgx_grad_norm(e, 1, P, None, need, None) == NULL
    assert lib.cgx_grad_norm(e, 1, P + 2, P, need, None) == ALIGN
    assert lib.cgx_grad_norm(e, 1, P, P + 8, need, None) == ALIGN
    assert lib.cgx_grad_norm(e, 1, P, P, need - 1, None) == SIZE
    assert lib.cgx_grad_clip(None, 1, P, 1.0, None, 0, None) == NULL
    assert lib.cgx_grad_clip(e, 1, None, 1.0, None, 0, None) == NULL
    assert lib.cgx_grad_clip(e, 1, P + 1, 1.0, None, 0, None) == ALIGN
    assert lib.cgx_grad_clip(e, 1, P, -1.0, None, 0, None) == SIZE
    assert lib.cgx_grad_clip(e, 1, P, float("nan"), None, 0, None) == SIZE
    assert lib.cgx_grad_clip(e, 1, P, 1.0, P, 3, None) == DTYPE
    assert lib.cgx_grad_clip(e, 1, P, 1.0, P + 4, 0, None) == ALIGN
    # nothing to scale: no launch
    assert lib.cgx_grad_clip(None, 0, P, 1.0, None, 0, None) == OK
    assert lib.cgx_grad_clip(entries((None, 0, 1, 0)), 1, P, 1.0, P, 0, None) == OK


def test_bfloat16_is_no_type_of_a_plan(lib):
    plan = cgx.Plan([0, 100], [4], 128, cgx.BF16)
    with pytest.raises(cgx.CgxError) as e:
        cgx.cgx_sizes(plan)
    assert e.value.status == DTYPE


def test_binding_refuses_what_the_kernels_would_overrun(lib):
    import torch

    class Fake:
        """A device tensor as far as the checks look."""
        is_cuda, device = True, "cuda:0"

        def __init__(self, shape, dtype, contiguous=True):
            self.shape, self.dtype, self.ndim, self._c = shape, dtype, len(shape), contiguous

        def numel(self): return int(np.prod(self.shape))
        def element_size(self): return torch.empty(0, dtype=self.dtype).element_size()
        def is_contiguous(self): return self._c
        def data_ptr(self): return P

    f, i = torch.float32, torch.int64
    good = dict(hidden=Fake((4, 64), f), weight=Fake((100, 64), f), targets=Fake((4,), i), loss=Fake((4,), f), lse=Fake((4,), f),
                workspace=Fake((8,), torch.uint8))

    def loss(**other):
        cgx.cgx_head_loss(**{**good, **other}, stream=0)

    with pytest.raises(cgx.CgxError):                       # everything passes up to the workspace's size
        loss()
    for other, word in ((dict(hidden=Fake((256,), f)), "matrix"), (dict(weight=Fake((100, 65), f)), "65"),
                        (dict(weight=Fake((100, 64), torch.float16)), "float16"), (dict(targets=Fake((5,), i)), "5 entries"),
                        (dict(targets=Fake((4,), torch.int32)), "int32"), (dict(loss=Fake((3,), f)), "12 bytes"),
                        (dict(lse=Fake((4,), torch.float64)), "float64"), (dict(hidden=Fake((4, 64), torch.float64)), "float64"),
                        (dict(hidden=Fake((4, 64), f, False)), "contiguous"), (dict(weight=Fake((100, 64), f, False)), "contiguous")):
        with pytest.raises(ValueError, match=word):
            loss(**other)
    grads = dict(hidden=good["hidden"], weight=good["weight"], targets=good["targets"], lse=good["lse"], dloss=Fake((4,), f),
                 dhidden=Fake((4, 64), f), dweight=Fake((100, 64), f), workspace=good["workspace"])
    with pytest.raises(cgx.CgxError):
        cgx.cgx_head_loss_grad(**grads, stream=0)
    for other, word in ((dict(dhidden=Fake((4, 63), f)), "bytes"), (dict(dweight=Fake((99, 64), f)), "bytes"),
                        (dict(dweight=Fake((100, 64), torch.bfloat16)), "bfloat16"), (dict(dloss=Fake((3,), f)), "bytes")):
        with pytest.raises(ValueError, match=word):
            cgx.cgx_head_loss_grad(**{**grads, **other})
    some = [Fake((4, 64), f), Fake((9,), torch.bfloat16)]
    with pytest.raises(ValueError, match="tensor 1.*int64"):
        cgx.cgx_grad_norm([some[0], Fake((9,), i)], Fake((1,), f), good["workspace"])
    with pytest.raises(ValueError, match="contiguous"):
        cgx.cgx_grad_norm([Fake((9, 9), f, False)], Fake((1,), f), good["workspace"])
    with pytest.raises(cgx.CgxError):
        cgx.cgx_grad_norm(some, Fake((1,), f), good["workspace"], stream=0)
    with pytest.raises(ValueError, match="norm"):
        cgx.cgx_grad_clip(some, Fake((1,), torch.float64), 1.0)
    with pytest.raises(ValueError, match="1056 bytes|1060"):
        cgx.cgx_grad_clip(some, Fake((1,), f), 1.0, out=Fake((264,), f))
    with pytest.raises(ValueError, match="out"):
        cgx.cgx_grad_clip(some, Fake((1,), f), 1.0, out=Fake((265,), torch.int64))
    with pytest.raises(ValueError, match="lives on|device"):
        cgx.cgx_grad_norm([torch.zeros(4)], Fake((1,), f), good["workspace"])


def test_head_sizes_a_launch_cannot_hold(lib):
    n = ctypes.c_size_t()
    for tokens, width, vocab in ((1 << 20, 64, 1 << 16), (1 << 20, 1 << 16, 100), ((1 << 24) - 1, 1 << 17, 1)):
        assert lib.cgx_head_workspace(tokens, width, vocab, 0, 1, ctypes.byref(n)) == SIZE
    assert lib.cgx_head_workspace(1 << 20, 4096, 50257, 2, 1, ctypes.byref(n)) == OK
    # pieces of the vocabulary stay small beside what a million tokens need themselves
    assert n.value < 2 * ((1 << 20) * 4096 * (2 + 4)) + (4 << 30)


def test_workspace_layout_is_clean_under_asan_and_ubsan(tmp_path):
    """The host code that lays the workspace out, with a driver that checks every section's place on many sizes."""
    import shutil
    import subprocess
    if not shutil.which("g++"):
        pytest.skip("needs g++")
    here = os.path.dirname(os.path.abspath(__file__))
    exe = str(tmp_path / "driver")
    subprocess.run(["g++", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-g", "-O1", "-std=c++17",
                    os.path.join(here, "host_sanitize", "head_layout.cpp"),
                    os.path.join(os.path.dirname(here), "paper_2111_08617_amd", "csrc", "cgx_head.cpp"), "-o", exe], check=True)
    run = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert run.returncode == 0 and "all checks passed" in run.stdout, (run.stdout[-2000:], run.stderr[-2000:])


def test_head_sizes_whose_last_tiles_make_the_launch_too_large(lib):
    """A grid has tiles of 64 columns: sizes are bounded after rounding up to these, or 65536 x 1048575 logits would be exactly 2^32 threads."""
    n = ctypes.c_size_t()
    for tokens, width, vocab in ((65536, 32, (1 << 20) - 1), (8192, 32, (1 << 23) - 1), (200, 32, (1 << 28) - 1), ((1 << 24) - 1, 4064, 1)):
        for dt in (cgx.F32, cgx.F16, cgx.BF16):
            assert lib.cgx_head_workspace(tokens, width, vocab, dt, 0, ctypes.byref(n)) == SIZE
            assert lib.cgx_head_loss(P, P, P, tokens, width, vocab, dt, -100, P, P, P, 1 << 60, None) == SIZE
            assert lib.cgx_head_loss_grad(P, P, P, P, P, tokens, width, vocab, dt, -100, P, P, P, 1 << 60, None) == SIZE
    for tokens, width, vocab in ((65536, 32, (1 << 20) - 64), (8192, 32, (1 << 23) - 64), (200, 32, (1 << 28) - 64), ((1 << 24) - 1, 4032, 1)):
        assert lib.cgx_head_workspace(tokens, width, vocab, 0, 0, ctypes.byref(n)) == OK


def test_head_limits_are_the_documented_ones(tmp_path):
    """head_layout's answer on sizes around every limit, under the host's sanitizers."""
    import shutil
    import subprocess
    if not shutil.which("g++"):
        pytest.skip("needs g++")
    here = os.path.dirname(os.path.abspath(__file__))
    exe = str(tmp_path / "driver")
    subprocess.run(["g++", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-g", "-O1", "-std=c++17",
                    os.path.join(here, "host_sanitize", "head_sizes.cpp"),
                    os.path.join(os.path.dirname(here), "paper_2111_08617_amd", "csrc", "cgx_head.cpp"), "-o", exe], check=True)
    run = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert run.returncode == 0 and "all checks passed" in run.stdout, (run.stdout[-2000:], run.stderr[-2000:])
    taken, refused = (int(w) for w in run.stdout.split() if w.isdigit())
    assert taken > 5000 and refused > 5000


def test_sizes_and_marks_that_the_c_types_cannot_hold(lib):
    """ctypes cuts an integer down to its argument's bits without a word: a width of 2^32 + 64 would be one of 64, an ignore mark of
    2^64 - 100 would be -100."""
    import torch

    class Fake:
        is_cuda, device, ndim = True, "cuda:0", 2

        def __init__(self, shape, dtype=torch.float32):
            self.shape, self.dtype, self.ndim = shape, dtype, len(shape)

        def numel(self): return int(np.prod([int(n) for n in self.shape], dtype=object))
        def element_size(self): return torch.empty(0, dtype=self.dtype).element_size()
        def is_contiguous(self): return True
        def data_ptr(self): return P

    for width in ((1 << 32) + 64, (1 << 31) + 64, -(1 << 32) + 64, 1 << 64):
        with pytest.raises(cgx.CgxError) as e:
            cgx.cgx_head_workspace(1, width, 100, cgx.F32)
        assert e.value.status == SIZE
    for tokens, vocab in (((1 << 64) + 1, 100), (1, (1 << 64) + 100), (1, -(1 << 64) + 100)):
        with pytest.raises(cgx.CgxError) as e:
            cgx.cgx_head_workspace(tokens, 64, vocab, cgx.F32)
        assert e.value.status == SIZE
    for dt in ((1 << 32), (1 << 32) + 2, -(1 << 32)):
        with pytest.raises(cgx.CgxError) as e:
            cgx.cgx_head_workspace(1, 64, 100, dt)
        assert e.value.status == DTYPE
    wide = (1 << 32) + 64
    args = dict(hidden=Fake((1, wide)), weight=Fake((100, wide)), targets=Fake((1,), torch.int64), lse=Fake((1,)), workspace=Fake((1 << 30,), torch.uint8))
    with pytest.raises(cgx.CgxError) as e:
        cgx.cgx_head_loss(**args, loss=Fake((1,)), stream=0)
    assert e.value.status == SIZE
    with pytest.raises(cgx.CgxError) as e:
        cgx.cgx_head_loss_grad(**args, dloss=Fake((1,)), dhidden=Fake((1, wide)), dweight=Fake((100, wide)), stream=0)
    assert e.value.status == SIZE
    args.update(hidden=Fake((1, 64)), weight=Fake((100, 64)), workspace=Fake((8,), torch.uint8))
    for mark in ((1 << 64) - 100, 1 << 63, -(1 << 63) - 1):
        with pytest.raises(ValueError, match="ignore"):
            cgx.cgx_head_loss(**args, loss=Fake((1,)), ignore=mark, stream=0)
        with pytest.raises(ValueError, match="ignore"):
            cgx.cgx_head_loss_grad(**args, dloss=Fake((1,)), dhidden=Fake((1, 64)), dweight=Fake((100, 64)), ignore=mark, stream=0)
    for mark in (-(1 << 63), (1 << 63) - 1):                 # these are int64 targets: the workspace is what is refused
        with pytest.raises(cgx.CgxError):
            cgx.cgx_head_loss(**args, loss=Fake((1,)), ignore=mark, stream=0)
