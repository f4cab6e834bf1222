"""What is made in a context is destroyed before it, once, in whatever order
Python lets go of the two (against a library that only writes its calls down)."""
import ctypes as C
import gc
from types import SimpleNamespace

import pytest

import paper_2609_18703_amd.ro as ro


class Written:
    """Stands for the library: creates handles, and notes what is destroyed."""

    def __init__(self):
        self.next, self.destroyed = 100, []

    def __getattr__(self, name):
        def call(*args):
            if name.endswith("_create"):
                out = C.cast(args[0] if name == "ro_ctx_create" else args[-1], C.POINTER(C.c_void_p))
                self.next += 1
                out[0] = self.next
            if name.endswith("_destroy"):
                self.destroyed.append(name)
            return 0
        return call


@pytest.fixture
def lib(monkeypatch):
    w = Written()
    monkeypatch.setattr(ro, "load", lambda path=None: w)
    return w


def make(lib):
    ctx = ro.Context(SimpleNamespace(cuda_stream=0))
    offsets = SimpleNamespace(is_cuda=True, is_contiguous=lambda: True, element_size=lambda: 8, numel=lambda: 3,
                              data_ptr=lambda: 8)
    return ctx, [ctx.chunk(1, 1, 1), ctx.grains(2), ctx.stream(offsets, 2)]


ALL = ["ro_chunk_destroy", "ro_grains_destroy", "ro_stream_destroy"]


def test_found_together_by_the_garbage_collector(lib):
    for _ in range(3):
        ctx, made = make(lib)
        ring = [ctx, *made]
        ring.append(ring)
        ctx.ring = ring
        del ctx, made, ring
        gc.collect()
        assert sorted(lib.destroyed[:3]) == ALL and lib.destroyed[3:] == ["ro_ctx_destroy"]
        lib.destroyed.clear()


@pytest.mark.parametrize("first", ["context", "made", "one of them"])
def test_closed_by_hand(lib, first):
    ctx, made = make(lib)
    if first == "made":
        for m in made:
            m.close()
            assert m.h is None
        assert lib.destroyed == ALL
    elif first == "one of them":
        made[1].close()
    ctx.close()
    assert sorted(lib.destroyed[:3]) == ALL and lib.destroyed[3:] == ["ro_ctx_destroy"]
    assert all(m.h is None for m in made)
    for m in made:
        m.close()
    ctx.close()
    del ctx, made, m
    gc.collect()
    assert len(lib.destroyed) == 4


def test_let_go_of_one_by_one(lib):
    ctx, made = make(lib)
    while made:
        made.pop()
    assert lib.destroyed == ALL[::-1] and not ctx._owned
    ctx, made = make(lib)
    lib.destroyed.clear()
    ctx.close()
    assert len(lib.destroyed) == 4


def test_nothing_is_owned_where_creation_fails(lib, monkeypatch):
    ctx, _ = make(lib)
    n = len(ctx._owned)
    monkeypatch.setattr(Written, "ro_chunk_create", lambda self, *a: ro.ECAP, raising=False)
    with pytest.raises(ro.RoError):
        ctx.chunk(1, 1, 1)
    gc.collect()
    assert len(ctx._owned) == n and lib.destroyed == []
