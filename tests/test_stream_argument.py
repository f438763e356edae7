"""``stream=`` of every call: what the call makes belongs to that stream, not to the caller's (CPU)."""
import contextlib
import inspect

import pytest
import torch
from torch.utils._python_dispatch import TorchDispatchMode

ca = pytest.importorskip("paper_2605_16839_amd")
from paper_2605_16839_amd import binding  # noqa: E402

MAKES = ("empty", "zeros", "full", "ones", "new_empty", "empty_like", "zeros_like", "fill_", "zero_")
STREAM = object()


class _Made(TorchDispatchMode):
    """Names of the operators that make or fill tensors, and the stream current at each."""

    def __init__(self, current):
        super().__init__()
        self.current, self.seen = current, []

    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        name = func.overloadpacket.__name__
        if name in MAKES:
            self.seen.append((name, self.current[-1]))
        return func(*args, **(kwargs or {}))


class _Library:
    """Stands for the shared library: every call succeeds, and every workspace is of 64 bytes."""

    def __init__(self, current):
        self.current, self.calls = current, []

    def __getattr__(self, name):
        if name.endswith("workspace_bytes"):
            return lambda *a: 64

        def call(*a):
            self.calls.append((name, self.current[-1]))
            return 0
        return call


@pytest.fixture
def world(monkeypatch):
    current = [None]

    @contextlib.contextmanager
    def stream(s):
        current.append(s)
        yield
        current.pop()

    lib = _Library(current)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(binding, "load", lambda *a: lib)
    monkeypatch.setattr(binding, "_stream", lambda *a: 0)
    monkeypatch.setattr(binding, "_here", lambda *a: (-1, 0))
    return current, lib


bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
f32 = lambda *s: torch.zeros(s)  # noqa: E731


def _calls():
    p = ca.Problem(1, 4, 2, 64, 64, 64, 3, [100], device=None)
    p.cached_len_dev = i32(1)
    c = ca.Cache(2, 4, 2, 64, 3, 9)
    q, pools, pt, masks = bf(1, 64, 4, 64), (bf(9, 64, 64), bf(9, 64, 64)), i32(1, 2, 3), torch.zeros(1, 4, 1, 1, dtype=torch.int64)
    T, rows = (i32(3), i32(6)), (i32(5), i32(12))
    table = i32(2, 2, 3)
    return {
        "pool_q_blocks": (p, q), "pool_k_blocks": (p, pools[0], pt), "block_scores": (p, f32(1), f32(1)),
        "select_blocks": (p, f32(1), 0.1), "estimate_masks": (p, q, pools[0], pt, 0.1),
        "estimate_masks_threshold": (p, q, pools[0], pt, 0.1, 1.0, 0.1),
        "select_blocks_threshold": (p, f32(1), 0.1, 1.0, 0.1), "build_block_tables": (p, masks, 2),
        "build_block_tables_noalloc": (p, masks, 2), "estimate_tables": (p, q, pools[0], pt, 0.1, 2),
        "chunk_attention": (p, q, pools, pt, T, 2, 0.1), "dense_paged_chunk_attention": (p, q, pools, pt, 0.1),
        "build_block_sparse_tables": (p, masks), "block_sparse_chunk_attention": (p, q, pools, pt, rows, 0.1),
        "gather_selected_pages": (p, pools, pt, T, 2), "packed_chunk_attention": (p, q, pools, T, 2, 0.1),
        "validate_tables": (p, 2, T),
        "assign_slots": (c, i32(2), 2, i32(2), table, i32(9), i32(1)),
        "release_pages": (c, i32(2), i32(2), table, i32(9), i32(1)),
        "rotary_append": (c, ca.Rotary(None), bf(2, 4, 64), bf(2, 2, 64), bf(2, 2, 64), i32(2),
                          torch.zeros(2, 2, dtype=torch.int64), pools),
        "decode_attention": (c, bf(2, 4, 64), pools, table, i32(2), 0.1),
    }


def test_every_call_with_a_stream_is_here():
    with_stream = {n for n in dir(ca) if inspect.isfunction(getattr(ca, n))
                   and "stream" in inspect.signature(getattr(ca, n)).parameters}
    assert with_stream == set(_calls())


@pytest.mark.parametrize("name", list(_calls()))
@pytest.mark.parametrize("by_place", [False, True])
def test_a_call_runs_under_its_stream(world, name, by_place):
    current, lib = world
    args, fn = _calls()[name], getattr(ca, name)
    for stream in (STREAM, None):
        lib.calls.clear()
        with _Made(current) as made:
            if by_place:
                n = len(inspect.signature(fn).parameters)
                rest = list(inspect.signature(fn).parameters.values())[len(args):n - 1]
                fn(*args, *[r.default for r in rest], stream)
            else:
                fn(*args, stream=stream)
        assert made.seen or name == "validate_tables"
        assert all(s is stream for _, s in made.seen), made.seen
        assert lib.calls and all(s is stream for _, s in lib.calls)
        assert current == [None]
