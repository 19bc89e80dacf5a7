"""Host-side tests of the head's calls that learn from a teacher's entries: sizes, refusals, the binding's checks.  No kernel is launched."""
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


def loss(lib, p=(P,) * 8, tokens=4, width=64, vocab=100, entries=5, dt=0, teacher=0, temperature=1.0, size=1 << 60):
    return lib.cgx_head_distill(*p[:4], tokens, width, vocab, entries, dt, teacher, -100, temperature, *p[4:], size, None)


def grad(lib, p=(P,) * 10, tokens=4, width=64, vocab=100, entries=5, dt=0, teacher=0, temperature=1.0, size=1 << 60):
    return lib.cgx_head_distill_grad(*p[:7], tokens, width, vocab, entries, dt, teacher, -100, temperature, *p[7:], size, None)


@pytest.mark.parametrize("sizes, want", [
    (dict(tokens=-1), SIZE), (dict(tokens=1 << 24), SIZE), (dict(width=0), SIZE), (dict(width=(1 << 17) + 1), SIZE), (dict(vocab=0), SIZE),
    (dict(vocab=1 << 31), SIZE), (dict(entries=0), SIZE), (dict(entries=-1), SIZE), (dict(entries=1025), SIZE), (dict(dt=3), DTYPE), (dict(dt=-1), DTYPE),
    (dict(tokens=1 << 20, vocab=1 << 16), SIZE)])
def test_sizes_that_are_refused(lib, sizes, want):
    n = ctypes.c_size_t()
    s = {**dict(tokens=4, width=64, vocab=100, entries=5, dt=0), **sizes}
    assert lib.cgx_head_distill_workspace(s["tokens"], s["width"], s["vocab"], s["entries"], s["dt"], 1, ctypes.byref(n)) == want
    assert loss(lib, **sizes) == want and grad(lib, **sizes) == want


def test_types_and_temperatures_that_are_refused(lib):
    for call in (loss, grad):
        for dt in (3, -1, 1 << 20):
            assert call(lib, teacher=dt) == DTYPE
        for t in (0.0, -1.0, float("nan"), float("inf"), 2.0**-10 * (1 - 2.0**-24), 2.0**10 * (1 + 2.0**-23), 2.0**-64, 2.0**64):
            assert call(lib, temperature=t) == SIZE
        for t in (2.0**-10, 2.0**10):                             # (these pass: the workspace is what is refused)
            assert call(lib, temperature=t, size=16) == SIZE and call(lib, (None,) * 10 if call is grad else (None,) * 8, temperature=t) == NULL


def test_pointers_that_are_refused(lib):
    n = ctypes.c_size_t()
    assert lib.cgx_head_distill_workspace(4, 64, 100, 5, 0, 1, None) == NULL
    for call, count, want_grad in ((loss, 8, 0), (grad, 10, 1)):
        for k in range(count):
            p = [P] * count
            p[k] = None
            assert call(lib, p) == NULL
            p[k] = ODD
            assert call(lib, p) == ALIGN
        p = [P] * count
        p[3] = P + 2                                              # a teacher of 16 bits may start there, one of 32 may not
        assert call(lib, p) == ALIGN
        assert lib.cgx_head_distill_workspace(4, 64, 100, 5, 0, want_grad, ctypes.byref(n)) == OK
        assert call(lib, size=n.value - 1) == SIZE
    # no tokens: nothing to do, nothing needed; a gradient is written all the same
    assert loss(lib, (None,) * 8, tokens=0, size=0) == OK
    assert grad(lib, (None,) * 10, tokens=0, size=0) == NULL


def test_workspace_sizes(lib):
    for dt in (cgx.F32, cgx.F16, cgx.BF16):
        for n, h, v, k in ((0, 1, 1, 1), (1, 1, 1, 1024), (3, 7, 11, 5), (4096, 768, 30522, 64)):
            assert 0 < cgx.cgx_head_distill_workspace(n, h, v, k, dt) <= cgx.cgx_head_distill_workspace(n, h, v, k, dt, True)
            # what the head needs, the operands of the gradient's products once more, and some numbers per token and entry: never the logits
            both = 2 * ((n + 511) + (v + 511)) * (h + 127) if dt == cgx.BF16 else 0
            assert cgx.cgx_head_distill_workspace(n, h, v, k, dt, True) <= cgx.cgx_head_workspace(n, h, v, dt, True) + both + n * (k * 16 + (v + 63) // 64 * 4 + 64) + 32768


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
    f, h, i = torch.float32, torch.float16, torch.int64
    both = dict(hidden=Fake((4, 64), f), weight=Fake((100, 64), f), ids=Fake((4, 5), i), teacher=Fake((4, 5), h), lse=Fake((4,), f), picked=Fake((4, 5), f),
                workspace=Fake((8,), torch.uint8))
    shared = ((dict(hidden=Fake((256,), f)), "matrix"), (dict(ids=Fake((20,), i)), "ids: a matrix"), (dict(teacher=Fake((20,), h)), "teacher: a matrix"),
              (dict(weight=Fake((100, 65), f)), "65"), (dict(weight=Fake((100, 64), h)), "float16"), (dict(ids=Fake((5, 5), i)), "5 rows for 4"),
              (dict(teacher=Fake((4, 6), h)), "logits for"), (dict(teacher=Fake((4, 5), i)), "teacher: element type"), (dict(ids=Fake((4, 5), torch.int32)), "int32"),
              (dict(hidden=Fake((4, 64), torch.float64)), "float64"), (dict(picked=Fake((4, 4), f)), "bytes"), (dict(picked=Fake((4, 5), h)), "float16"),
              (dict(lse=Fake((3,), f)), "bytes"), (dict(teacher=Fake((4, 5), h, False)), "contiguous"), (dict(ids=Fake((4, 5), i, False)), "contiguous"),
              (dict(teacher=Fake((4, 5), h, index=1)), "teacher.*current device"), (dict(workspace=Fake((8,), f, index=1)), "workspace.*current device"))
    for call, more, cases in ((cgx.cgx_head_distill, dict(loss=Fake((4,), f)), ((dict(loss=Fake((3,), f)), "bytes"),)),
                              (cgx.cgx_head_distill_grad, dict(dloss=Fake((4,), f), dhidden=Fake((4, 64), f), dweight=Fake((100, 64), f)),
                               ((dict(dloss=Fake((3,), f)), "bytes"), (dict(dhidden=Fake((4, 63), f)), "bytes"), (dict(dweight=Fake((99, 64), f)), "bytes"),
                                (dict(dweight=Fake((100, 64), torch.bfloat16)), "bfloat16")))):
        good = {**both, **more}
        with pytest.raises(cgx.CgxError) as e:                    # everything passes up to the workspace's size
            call(**good, stream=0)
        assert e.value.status == SIZE
        for other, word in shared + cases:
            with pytest.raises(ValueError, match=word):
                call(**{**good, **other}, stream=0)
        for mark in ((1 << 64) - 100, 1 << 63, -(1 << 63) - 1):
            with pytest.raises(ValueError, match="ignore"):
                call(**good, ignore=mark, stream=0)
        good["workspace"] = Fake((1 << 40,), torch.uint8)
        for t in (0.0, -2.0, float("nan")):
            with pytest.raises(cgx.CgxError):
                call(**good, temperature=t, stream=0)
    for sizes, dt in (((1, (1 << 32) + 64, 100, 5), 0), ((1, 64, 100, (1 << 32) + 5), 0), (((1 << 64) + 1, 64, 100, 5), 0)):
        with pytest.raises(cgx.CgxError) as e:
            cgx.cgx_head_distill_workspace(*sizes, dt)
        assert e.value.status == SIZE
