"""Tests that give a call a stream of its own order its work against the fills on the current one (conftest.py); no GPU."""
import ast
import glob
import os
import types

import conftest
import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


class Stream:
    def __init__(self, name, log):
        self.name, self.log = name, log

    def wait_stream(self, other):
        self.log.append(f"{self.name} waits for {other.name}")


def test_a_call_comes_after_what_is_queued_and_ahead_of_what_follows():
    log = []
    current, side = Stream("current", log), Stream("side", log)

    def call(x, out=None, stream=None):
        log.append(f"call {x} {out} on {stream.name if stream else 'current'}")
        if x == 3:
            raise ValueError("refused")

    ordered = conftest.in_order(call, lambda: current)
    ordered(1, out=2)
    assert log == ["call 1 2 on current"]
    del log[:]
    ordered(1, out=2, stream=side)
    assert log == ["side waits for current", "call 1 2 on side", "current waits for side"]
    with pytest.raises(ValueError):
        ordered(3, stream=side)


def test_every_call_of_a_module_that_takes_a_stream_is_ordered(monkeypatch):
    log = []
    current, side = Stream("current", log), Stream("side", log)
    module = types.ModuleType("module")
    exec("def cgx_a(x, stream=None): return x\ndef cgx_b(x): return x\ndef other(stream=None): return 5\n", module.__dict__)
    with monkeypatch.context() as m:
        conftest.order_calls(m, module, lambda: current)
        assert module.cgx_a(1, stream=side) == 1 and module.cgx_b(2) == 2 and module.other(stream=side) == 5
    assert log == ["side waits for current", "current waits for side"]
    assert module.cgx_a(1, stream=side) == 1 and len(log) == 2


def test_all_tests_whose_helpers_take_a_stream_are_ordered():
    """A helper fills what it gives to a call; a test that hands it a stream has to be in the list, and the list names tests that exist."""
    found = set()
    for path in glob.glob(os.path.join(HERE, "test_gpu_*.py")):
        functions = [n for n in ast.parse(open(path).read()).body if isinstance(n, ast.FunctionDef)]
        helpers = {f.name for f in functions if not f.name.startswith("test_") and "stream" in [a.arg for a in f.args.args + f.args.kwonlyargs]}
        for f in functions:
            for n in ast.walk(f):
                if f.name.startswith("test_") and isinstance(n, ast.Call) and isinstance(n.func, ast.Name) and n.func.id in helpers \
                        and any(k.arg == "stream" for k in n.keywords):
                    found.add((os.path.basename(path), f.name))
    assert found == conftest.ON_OTHER_STREAMS


def test_an_ordered_test_sees_ordered_calls(monkeypatch):
    """What the fixture does for one of them, and not for this one."""
    from paper_2111_08617_amd import binding
    before = binding.cgx_embed
    assert not hasattr(before, "__wrapped__")
    node = types.SimpleNamespace(path=types.SimpleNamespace(name="test_gpu_embed.py"), originalname="test_on_another_stream")
    with monkeypatch.context() as m:
        conftest.order_where_needed(node, m)
        assert binding.cgx_embed.__wrapped__ is before and binding.cgx_grad_norm.__wrapped__ and binding.cgx_head_loss.__wrapped__
    assert binding.cgx_embed is before
