"""What the calls of requests that share pages, and the norms of heads, refuse before anything is
enqueued; and ``stream=`` of those calls (CPU)."""
import contextlib
import inspect

import pytest
import torch

ca = pytest.importorskip("paper_2605_16839_amd")
from paper_2605_16839_amd import binding, sharing  # noqa: E402

FAKE = 0x1000    # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def lib():
    return ca.load()


def _cache(**kw):
    base = dict(batch=2, num_q_heads=8, num_kv_heads=2, head_dim=128, max_kv_blocks=16, num_pages=99)
    base.update(kw)
    return ca.Cache(**base)


def _name(lib, status):
    return lib.ca_status_string(status).decode()


FORK = ("parent", "keep", "seq", "table", "shares", "free", "cap", "count", "k", "v", "seq_out", "table_out",
        "shares_out", "free_out", "count_out", "ws", "nbytes")
COMPACT = ("seq", "table", "shares", "free", "cap", "count", "k", "v", "new_page", "table_out", "shares_out",
           "free_out", "count_out", "ws", "nbytes")
PREFIX = ("q", "k", "v", "table", "len", "share", "share_len", "shares", "scale", "out", "lse", "ws", "nbytes")


def _call(lib, fn, names, c, **kw):
    a = dict({n: FAKE for n in names}, cap=99, nbytes=1 << 40, shares_=0)
    if "scale" in names:
        a.update(shares=3, scale=0.1)
    a.update(kw)
    return _name(lib, fn(c, *[a[n] for n in names], None))


@pytest.mark.parametrize("kw,code", [
    (dict(cap=98), "CA_ERR_SHAPE"), (dict(cap=-1), "CA_ERR_SHAPE"), (dict(k=FAKE + 8), "CA_ERR_UNALIGNED"),
    (dict(v=FAKE + 2), "CA_ERR_UNALIGNED"), (dict(ws=None), "CA_ERR_WORKSPACE"),
    (dict(ws=FAKE + 8), "CA_ERR_WORKSPACE"), (dict(nbytes=64), "CA_ERR_WORKSPACE"),
] + [({n: None}, "CA_ERR_NULL") for n in FORK if n not in ("keep", "cap", "ws", "nbytes")])
def test_fork_refuses(lib, kw, code):
    assert _call(lib, lib.ca_fork_requests, FORK, _cache().ref, **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(cap=98), "CA_ERR_SHAPE"), (dict(k=FAKE + 8), "CA_ERR_UNALIGNED"), (dict(ws=None), "CA_ERR_WORKSPACE"),
    (dict(ws=FAKE + 4), "CA_ERR_WORKSPACE"), (dict(nbytes=64), "CA_ERR_WORKSPACE"),
    (dict(shares=None), "CA_ERR_NULL"), (dict(shares_out=None), "CA_ERR_NULL"),
] + [({n: None}, "CA_ERR_NULL") for n in COMPACT if n not in ("shares", "shares_out", "cap", "ws", "nbytes")])
def test_compact_refuses(lib, kw, code):
    assert _call(lib, lib.ca_compact_pages, COMPACT, _cache().ref, **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(scale=0.0), "CA_ERR_SHAPE"), (dict(scale=float("nan")), "CA_ERR_SHAPE"),
    (dict(scale=float("inf")), "CA_ERR_SHAPE"), (dict(shares=-1), "CA_ERR_SHAPE"),
    (dict(shares=513), "CA_ERR_UNSUPPORTED"), (dict(q=FAKE + 8), "CA_ERR_UNALIGNED"),
    (dict(out=FAKE + 2), "CA_ERR_UNALIGNED"), (dict(k=FAKE + 8), "CA_ERR_UNALIGNED"),
    (dict(ws=None), "CA_ERR_WORKSPACE"), (dict(ws=FAKE + 8), "CA_ERR_WORKSPACE"),
    (dict(nbytes=8), "CA_ERR_WORKSPACE"), (dict(share=None), "CA_ERR_NULL"), (dict(share_len=None), "CA_ERR_NULL"),
    (dict(shares=0, share=None, share_len=None, ws=None), "CA_ERR_WORKSPACE"),     # the next check
] + [({n: None}, "CA_ERR_NULL") for n in ("q", "k", "v", "table", "len", "out")])
def test_prefix_refuses(lib, kw, code):
    assert _call(lib, lib.ca_prefix_decode_attention, PREFIX, _cache().ref, **kw) == code


def test_prefix_refuses_sizes(lib):
    def status(**kw):
        return _call(lib, lib.ca_prefix_decode_attention, PREFIX, _cache(**kw).ref, ws=None)
    assert status(batch=2049) == "CA_ERR_UNSUPPORTED" and status(batch=2048) == "CA_ERR_WORKSPACE"
    assert status(batch=2048, max_kv_blocks=16384, num_q_heads=64, num_kv_heads=64) == "CA_ERR_SHAPE"
    assert status(batch=2047, max_kv_blocks=16384, num_q_heads=64, num_kv_heads=64) == "CA_ERR_WORKSPACE"
    assert status(batch=2047, max_kv_blocks=16384, num_q_heads=32 * 257, num_kv_heads=32) == "CA_ERR_WORKSPACE"
    assert status(batch=2047, max_kv_blocks=16384, num_q_heads=64 * 257, num_kv_heads=64) == "CA_ERR_SHAPE"


def test_null_and_bad_caches(lib):
    for c in (None, _cache(head_dim=96).ref, _cache(batch=0).ref):
        assert lib.ca_fork_workspace_bytes(c) == 0 and lib.ca_compact_workspace_bytes(c) == 0
        assert lib.ca_prefix_decode_workspace_bytes(c, 1) == 0
        for fn, names in ((lib.ca_fork_requests, FORK), (lib.ca_compact_pages, COMPACT),
                          (lib.ca_prefix_decode_attention, PREFIX)):
            assert _call(lib, fn, names, c) in ("CA_ERR_NULL", "CA_ERR_UNSUPPORTED", "CA_ERR_SHAPE")
    assert lib.ca_prefix_decode_workspace_bytes(_cache().ref, -1) == 0
    assert lib.ca_prefix_decode_workspace_bytes(_cache().ref, 513) == 0
    assert lib.ca_prefix_decode_workspace_bytes(_cache().ref, 0) > 0


def _norm(lib, n, T=3, c=None, rot=None):
    r = rot or ca.Rotary(None)
    return _name(lib, lib.ca_norm_rotary_append(c or _cache().ref, r.ref, n, T, FAKE, 1024, FAKE, 256, FAKE, 256,
                                                FAKE, FAKE, None, FAKE, FAKE, None))


def test_norm_refuses(lib):
    def norm(q=FAKE, k=FAKE, eps=1e-6):
        n = ca.HeadNorm(None, None, eps=eps)
        n.c.q_weight, n.c.k_weight = q, k
        return n.ref
    assert _norm(lib, None) == "CA_ERR_NULL"
    for eps in (-1e-6, float("nan"), float("inf")):
        assert _norm(lib, norm(eps=eps)) == "CA_ERR_SHAPE"
    assert _norm(lib, norm(q=FAKE + 8)) == "CA_ERR_UNALIGNED"
    assert _norm(lib, norm(k=FAKE + 4)) == "CA_ERR_UNALIGNED"
    assert _norm(lib, norm()) == "CA_ERR_NULL"                    # q_out
    assert _norm(lib, norm(q=None, k=None, eps=0.0), T=0) == "CA_OK"
    assert _norm(lib, norm(), T=-1) == "CA_ERR_SHAPE" and _norm(lib, norm(), c=_cache(head_dim=96).ref) == "CA_ERR_UNSUPPORTED"


def test_head_norm_refuses():
    w = torch.ones(128)
    for q, k in ((w, w.bfloat16()), (w, w[:64]), (w.double(), None), (w.view(2, 64), None)):
        with pytest.raises(ValueError):
            ca.HeadNorm(q, k)
    with pytest.raises(ValueError, match="contiguous"):
        ca.HeadNorm(torch.ones(256)[::2], None)
    assert ca.HeadNorm(None, None).head_dim is None and ca.HeadNorm(None, w).c.weight_fp32 == 1


def test_binding_refuses_the_cpu():
    c = _cache()
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    pools = (torch.zeros(99, 64, 128, dtype=torch.bfloat16),) * 2
    state = (i32(2), i32(2, 2, 16), i32(99), i32(99), i32(1))
    for call in (lambda: sharing.fork_requests(c, i32(2), *state, pools),
                 lambda: sharing.compact_pages(c, *state, pools),
                 lambda: sharing.prefix_decode_attention(c, pools[0][:2, :8], pools, state[1], i32(2), i32(2), i32(1), 0.1)):
        with pytest.raises(ValueError, match="current device"):
            call()


# ---------------------------------------------------------------------------
# stream=: what a call makes belongs to that stream
# ---------------------------------------------------------------------------
def _calls():
    c = ca.Cache(2, 4, 2, 64, 3, 9)
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    pools = (bf(9, 64, 64), bf(9, 64, 64))
    state = (i32(2), i32(2, 2, 3), i32(9), i32(9), i32(1))
    return {"fork_requests": (c, i32(2), *state, pools), "compact_pages": (c, *state, pools),
            "prefix_decode_attention": (c, bf(2, 4, 64), pools, state[1], i32(2), i32(2), i32(1), 0.1)}


def test_every_call_of_the_module_is_here():
    with_stream = {n for n in sharing.__all__ if "stream" in inspect.signature(getattr(sharing, n)).parameters}
    assert with_stream == set(_calls())
    public = {n for n in dir(sharing) if inspect.isfunction(getattr(sharing, n)) and not n.startswith("_")
              and getattr(sharing, n).__module__ == sharing.__name__}
    assert public == set(sharing.__all__)


@pytest.mark.parametrize("name", list(_calls()))
def test_a_call_runs_under_its_stream(monkeypatch, name):
    current, made, called = [None], [], []

    @contextlib.contextmanager
    def stream(s):
        current.append(s)
        yield
        current.pop()

    class Library:
        def __getattr__(self, n):
            return (lambda *a: 64) if n.endswith("workspace_bytes") else lambda *a: called.append(current[-1]) or 0

    monkeypatch.setattr(torch.cuda, "stream", stream)
    for m in (binding, sharing):
        monkeypatch.setattr(m, "load", lambda *a: Library())
    monkeypatch.setattr(sharing, "_here", lambda *a: (-1, 0))
    for n in ("empty", "full", "empty_like"):
        monkeypatch.setattr(sharing.torch, n, lambda *a, f=getattr(torch, n), **k: made.append(current[-1]) or f(*a, **k))
    args, fn, mark = _calls()[name], getattr(sharing, name), object()
    for s in (mark, None):
        made.clear(), called.clear()
        fn(*args, stream=s)
        assert made and all(x is s for x in made) and called == [s] and current == [None]
    n = len(inspect.signature(fn).parameters)
    rest = [p.default for p in list(inspect.signature(fn).parameters.values())[len(args):n - 1]]
    called.clear()
    fn(*args, *rest, mark)
    assert called == [mark]


def test_fork_refuses_more_rows_than_a_launch_has_workgroups(lib):
    """Its second launch has 256 threads for every row, and a launch fewer than 2^32."""
    most = dict(num_q_heads=1, num_kv_heads=1, max_kv_blocks=1)
    for batch, code in ((1 << 24, "CA_ERR_UNSUPPORTED"), ((1 << 24) - 1, "CA_ERR_WORKSPACE")):
        c = _cache(batch=batch, **most)
        assert _call(lib, lib.ca_fork_requests, FORK, c.ref, ws=None) == code
        assert (lib.ca_fork_workspace_bytes(c.ref) == 0) == (code == "CA_ERR_UNSUPPORTED")
