import functools
import inspect
import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a real MI355X (run with -m gpu)")


@pytest.fixture(scope="session")
def oracle():
    import oracle as _oracle
    _oracle.build()
    return _oracle


# Tests whose helpers fill workspaces and outputs on the current stream and then give a call another stream (`stream=`):
# without an order between the two a fill could still run, or already run again, while the call's kernels use what it fills.
ON_OTHER_STREAMS = {("test_gpu_distill.py", "test_on_another_stream"), ("test_gpu_embed.py", "test_on_another_stream"),
                    ("test_gpu_head.py", "test_same_call_same_bits_and_other_streams"), ("test_gpu_grad.py", "test_streams_and_graphs")}


def in_order(call, current_stream):
    """`call`, whose work on a stream of its own comes after all that is queued on the current stream before it, and ahead of
    all that is queued behind it."""
    @functools.wraps(call)
    def ordered(*args, stream=None, **kwargs):
        if stream is None:
            return call(*args, **kwargs)
        current = current_stream()
        stream.wait_stream(current)
        try:
            return call(*args, stream=stream, **kwargs)
        finally:
            current.wait_stream(stream)
    return ordered


def order_calls(monkeypatch, module, current_stream):
    """Every function of `module` that takes a stream, in order (until the test has ended)."""
    for name, f in inspect.getmembers(module, inspect.isfunction):
        if name.startswith("cgx_") and "stream" in inspect.signature(f).parameters:
            monkeypatch.setattr(module, name, in_order(f, current_stream))


def order_where_needed(node, monkeypatch):
    if (node.path.name, getattr(node, "originalname", None)) in ON_OTHER_STREAMS:
        import torch
        from paper_2111_08617_amd import binding
        order_calls(monkeypatch, binding, torch.cuda.current_stream)


@pytest.fixture(autouse=True)
def calls_on_other_streams_in_order(request, monkeypatch):
    order_where_needed(request.node, monkeypatch)
