"""Host-side tests of the embedding's calls: sizes, refusals, the binding's checks.  No kernel is launched."""
import ctypes
import os

import numpy as np
import pytest

from paper_2111_08617_amd import binding as cgx

P, ODD = 0x10000, 0x10001          # addresses that pass and fail the alignment checks; nothing is read before a refusal
OK, NULL, SIZE, DTYPE, ALIGN = 0, -1, -2, -7, -9


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(cgx.LIB_PATH):
        from paper_2111_08617_amd import build
        build.build()
    return cgx.lib()


@pytest.mark.parametrize("tokens, width, vocab, dt, want", [
    (-1, 64, 100, 0, SIZE), (1 << 24, 64, 100, 0, SIZE), (1, 0, 100, 0, SIZE), (1, -5, 100, 0, SIZE), (1, (1 << 17) + 1, 100, 0, SIZE),
    (1, 64, 0, 0, SIZE), (1, 1, 1 << 28, 0, SIZE), (1, 64, 100, 3, DTYPE), (1, 64, 100, -1, DTYPE), (1, 1 << 17, 1 << 18, 2, SIZE),
    ((1 << 24) - 1, 1 << 12, 5, 2, SIZE), (1, 64, 1 << 62, 0, SIZE)])
def test_sizes_that_are_refused(lib, tokens, width, vocab, dt, want):
    n = ctypes.c_size_t()
    assert lib.cgx_embed(P, P, tokens, width, vocab, dt, -100, 1.0, P, None) == want
    assert lib.cgx_embed_grad_workspace(tokens, width, vocab, dt, ctypes.byref(n)) == want
    assert lib.cgx_embed_grad(P, P, tokens, width, vocab, dt, -100, 1.0, 0, P, P, 1 << 60, None) == want


def test_sizes_that_are_taken(lib):
    for dt in (cgx.F32, cgx.F16, cgx.BF16):
        for n, h, v in ((0, 1, 1), (1, 1, 1), (3, 7, 11), (8192, 2048, 50257), ((1 << 24) - 1, 2047, 300), (5, 127, (1 << 28) - 1), (9, 1 << 17, (1 << 18) - 1)):
            assert cgx.cgx_embed_grad_workspace(n, h, v, dt) > 0
    # lists of tokens, and parts of rows: far below the table's gradient and that of the rows
    assert cgx.cgx_embed_grad_workspace(8192, 2048, 50257, cgx.BF16) < 8192 * 2048 * 2


def test_pointers_that_are_refused(lib):
    n = ctypes.c_size_t()
    assert lib.cgx_embed_grad_workspace(4, 64, 100, 0, None) == NULL
    assert lib.cgx_embed_grad_workspace(4, 64, 100, 0, ctypes.byref(n)) == OK
    for bad, want in ((None, NULL), (ODD, ALIGN)):
        for k in range(3):
            a = [P] * 3
            a[k] = bad
            assert lib.cgx_embed(a[0], a[1], 4, 64, 100, 0, -100, 1.0, a[2], None) == want
        for k in range(4):
            a = [P] * 4
            a[k] = bad
            assert lib.cgx_embed_grad(a[0], a[1], 4, 64, 100, 0, -100, 1.0, 0, a[2], a[3], 1 << 60, None) == want
    assert lib.cgx_embed(P + 8, P, 4, 64, 100, 0, -100, 1.0, P, None) == ALIGN
    assert lib.cgx_embed_grad(P, P, 4, 64, 100, 0, -100, 1.0, 0, P, P, n.value - 1, None) == SIZE
    # no tokens: nothing to look up, nothing to add; a gradient that is not added is written
    assert lib.cgx_embed(None, None, 0, 64, 100, 0, -100, 1.0, None, None) == OK
    assert lib.cgx_embed_grad(None, None, 0, 64, 100, 0, -100, 1.0, 1, P, P, 1 << 60, None) == OK
    assert lib.cgx_embed_grad(None, None, 0, 64, 100, 0, -100, 1.0, 0, None, None, 0, None) == NULL


class Fake:
    """A device tensor as far as the checks look."""
    is_cuda, device = True, "cuda:0"

    def __init__(self, shape, dtype, contiguous=True, index=0):
        self.shape, self.dtype, self.ndim, self._c, self._index = shape, dtype, len(shape), contiguous, index

    def numel(self): return int(np.prod([int(n) for n in self.shape], dtype=object))
    def element_size(self):
        import torch
        return torch.empty(0, dtype=self.dtype).element_size()
    def is_contiguous(self): return self._c
    def data_ptr(self): return P
    def get_device(self): return self._index


def test_binding_refuses_what_the_kernels_would_overrun(lib):
    import torch
    f, i = torch.float32, torch.int64
    rows = dict(table=Fake((100, 64), f), ids=Fake((4,), i), out=Fake((4, 64), f))
    grads = dict(dout=Fake((4, 64), f), ids=Fake((4,), i), dtable=Fake((100, 64), f), workspace=Fake((8,), torch.uint8))
    for call, good, cases in (
            (cgx.cgx_embed, rows, ((dict(table=Fake((6400,), f)), "matrix"), (dict(out=Fake((256,), f)), "matrix"), (dict(out=Fake((4, 65), f)), "65"),
                                   (dict(out=Fake((4, 64), torch.float16)), "float16"), (dict(table=Fake((100, 64), torch.float64)), "float64"),
                                   (dict(ids=Fake((5,), i)), "5 entries"), (dict(ids=Fake((4,), torch.int32)), "int32"),
                                   (dict(table=Fake((100, 64), f, False)), "contiguous"), (dict(out=Fake((4, 64), f, index=1)), "current device"))),
            (cgx.cgx_embed_grad, grads, ((dict(dtable=Fake((6400,), f)), "matrix"), (dict(dout=Fake((4, 65), f)), "65"), (dict(ids=Fake((3,), i)), "3 entries"),
                                         (dict(dout=Fake((4, 64), torch.bfloat16)), "bfloat16"), (dict(dtable=Fake((100, 64), i)), "int64"),
                                         (dict(dout=Fake((4, 64), f, False)), "contiguous"), (dict(workspace=Fake((8,), f, index=2)), "current device")))):
        for other, word in cases:
            with pytest.raises(ValueError, match=word):
                call(**{**good, **other}, stream=0)
        for mark in ((1 << 64) - 100, 1 << 63, -(1 << 63) - 1):
            with pytest.raises(ValueError, match="ignore"):
                call(**good, ignore=mark, stream=0)
    with pytest.raises(cgx.CgxError) as e:                  # everything passes up to the workspace's size
        cgx.cgx_embed_grad(**grads, stream=0)
    assert e.value.status == SIZE
    wide = (1 << 32) + 64
    with pytest.raises(cgx.CgxError) as e:
        cgx.cgx_embed(Fake((100, wide), f), Fake((1,), i), Fake((1, wide), f), stream=0)
    assert e.value.status == SIZE
    for sizes in (((1 << 64) + 1, 64, 100), (1, (1 << 32) + 64, 100), (1, 64, (1 << 64) + 100)):
        with pytest.raises(cgx.CgxError) as e:
            cgx.cgx_embed_grad_workspace(*sizes, cgx.F32)
        assert e.value.status == SIZE


def test_workspaces_are_clean_under_asan_and_ubsan(tmp_path):
    """The host code that lays out the workspaces of these calls and of distillation, on many sizes."""
    import shutil
    import subprocess
    if not shutil.which("g++"):
        pytest.skip("needs g++")
    here = os.path.dirname(os.path.abspath(__file__))
    csrc = os.path.join(os.path.dirname(here), "paper_2111_08617_amd", "csrc")
    exe = str(tmp_path / "driver")
    subprocess.run(["g++", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-g", "-O1", "-std=c++17",
                    os.path.join(here, "host_sanitize", "more_layouts.cpp"),
                    *(os.path.join(csrc, f) for f in ("cgx_embed.cpp", "cgx_distill.cpp", "cgx_head.cpp")), "-o", exe], check=True)
    run = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert run.returncode == 0 and "all checks passed" in run.stdout, (run.stdout[-2000:], run.stderr[-2000:])
    taken, refused = (int(w) for w in run.stdout.split() if w.isdigit())
    assert taken > 5000 and refused > 5000
