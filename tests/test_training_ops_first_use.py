"""The tensor forms' first use, from several threads and after a failed load: no GPU needed."""
import threading

import pytest
import torch

from paper_2602_17254_b200 import binding as B
from paper_2602_17254_b200 import build


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def _first_use(x):
    with pytest.raises(ValueError):                 # a CPU tensor: refused behind the load
        B._stream_of(x)


def test_no_thread_passes_before_the_library_is_there(monkeypatch):
    real, entered, go = B.lib, threading.Event(), threading.Event()
    monkeypatch.setattr(B, "_lib", None)
    monkeypatch.setattr(B, "_torch", None)

    def slow():
        entered.set()
        assert go.wait(30)
        return real()

    monkeypatch.setattr(B, "lib", slow)
    seen = []

    def use():
        _first_use(torch.zeros(2))
        seen.append(B._lib)

    threads = [threading.Thread(target=use) for _ in range(3)]
    threads[0].start()
    assert entered.wait(30)                         # the first thread is inside the load ...
    for t in threads[1:]:
        t.start()
    for t in threads[1:]:
        t.join(0.2)                                 # ... and the others have had time to run past it
    go.set()
    for t in threads:
        t.join(30)
    assert len(seen) == 3 and all(s is not None for s in seen)


def test_a_failed_load_is_tried_again(monkeypatch):
    monkeypatch.setattr(B, "_lib", None)
    monkeypatch.setattr(B, "_torch", None)
    path = B.LIB_PATH
    monkeypatch.setattr(B, "LIB_PATH", path + ".missing")
    for _ in range(2):
        with pytest.raises(RuntimeError, match="missing"):
            B._stream_of(torch.zeros(2))
    monkeypatch.setattr(B, "LIB_PATH", path)
    _first_use(torch.zeros(2))
    assert B._lib is not None


def test_type_codes_filled_by_another_thread_between_two_looks(monkeypatch):
    class Filled(dict):
        def get(self, key, default=None):
            was = super().get(key, default)
            super().update({torch.float32: B.FLOAT32, torch.bfloat16: B.BFLOAT16, torch.float16: B.FLOAT16})
            return was

    monkeypatch.setattr(B, "_FLOAT_CODES", Filled())
    assert B._float_code(torch.zeros(1), "x") == B.FLOAT32
    with pytest.raises(TypeError):
        B._float_code(torch.zeros(1, dtype=torch.int32), "x")
