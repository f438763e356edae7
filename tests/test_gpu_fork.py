"""Forks of requests and compaction of a pool against the oracle: every number exactly, every page
of the pools bit for bit."""
import numpy as np
import pytest
import torch

from _helpers import i32_dev
from oracle import serving, sharing

pytestmark = pytest.mark.gpu

ca = pytest.importorskip("paper_2605_16839_amd")
DEV = "cuda"
NAMES = ("seq_len", "page_table", "page_shares", "free_pages", "free_count")


def _state(rng, B, H, most, pages, steps=3, grow=90):
    """Requests that have grown and forked for some steps."""
    table, lens = np.full((B, H, most), -1), np.zeros(B, dtype=np.int64)
    shares, free = np.zeros(pages, dtype=np.int64), list(rng.permutation(pages))
    for i in range(steps):
        new = np.minimum(rng.integers(0, grow, B), 64 * most - lens)
        a = serving.assign_slots(new, int(new.sum()), lens, table, free, pages)
        if i == steps - 1:
            return a["seq_len"], a["page_table"], shares, a["free"]
        s = sharing.fork_requests(rng.integers(-1, B, B), None, a["seq_len"], a["page_table"], shares, a["free"], pages)
        lens, table, shares, free = s["seq_len"], s["page_table"], s["page_shares"], s["free"]


def _pools(rng, pages, D):
    return tuple(torch.from_numpy(rng.integers(-2**15, 2**15, (pages, 64, D)).astype(np.int16)).to(DEV).view(torch.bfloat16)
                 for _ in "kv")


def _devs(lens, table, shares, free, pages):
    fp = np.full(pages, -3)
    fp[:len(free)] = free
    return dict(zip(NAMES, (i32_dev(lens), i32_dev(table), i32_dev(shares), i32_dev(fp), i32_dev([len(free)]))))


def _check_fork(rng, parent, keep, lens, table, shares, free, pages, D=64, in_place=False, twice=True):
    B, H, most = table.shape
    want = sharing.fork_requests(parent, keep, lens, table, shares, free, pages)
    c = ca.Cache(B, H, H, D, most, pages)
    pools = _pools(rng, pages, D)
    before = [p.clone() for p in pools]
    ws = torch.full((ca.sharing.fork_workspace_bytes(c),), 0x5a, dtype=torch.uint8, device=DEV)
    d = _devs(lens, table, shares, free, pages)
    after = {n: torch.full_like(d[n], -3) for n in NAMES}
    if in_place is True:
        after = dict(d)
    elif in_place:
        after[in_place] = d[in_place]
    given = {n: t.clone() for n, t in d.items()}
    # out of place the call may be made again
    for _ in range(2 if twice and not in_place else 1):
        got = ca.sharing.fork_requests(c, i32_dev(parent), *[d[n] for n in NAMES], pools,
                                       keep_len=None if keep is None else i32_dev(keep), bufs=after, ws=ws)
        assert got is after
    torch.cuda.synchronize()
    assert np.array_equal(after["seq_len"].cpu().numpy(), want["seq_len"])
    live = np.arange(most)[None, None, :] < -(-want["seq_len"] // 64)[:, None, None]
    live = np.broadcast_to(live, table.shape)
    t = after["page_table"].cpu().numpy()
    assert np.array_equal(t[live], want["page_table"][live])
    assert (t[~live] == (table[~live] if in_place in (True, "page_table") else -3)).all()     # left alone
    assert np.array_equal(after["page_shares"].cpu().numpy(), want["page_shares"])
    n = len(want["free"])
    assert int(after["free_count"]) == n
    f = after["free_pages"].cpu().numpy()
    assert f[:n].tolist() == want["free"]
    if in_place not in (True, "free_pages"):
        assert (f[n:] == -3).all()
    for x in NAMES:
        if after[x] is not d[x]:
            assert torch.equal(d[x], given[x]), x
    for p, b in zip(pools, before):
        for x, y in want["copies"]:
            b[y] = b[x]
        assert torch.equal(p.view(torch.int16), b.view(torch.int16))
    return want


@pytest.mark.parametrize("in_place", [False, True, "page_table", "page_shares", "free_pages", "seq_len"])
@pytest.mark.parametrize("B,H,most,cut", [
    (1, 1, 1, False), (2, 1, 3, False), (7, 8, 9, False), (7, 3, 9, True), (64, 2, 7, False), (64, 8, 6, True),
    (300, 1, 5, True), (513, 2, 4, False), (5, 700, 3, True),
])
def test_fork(B, H, most, cut, in_place):
    rng = np.random.default_rng(B * 7 + H)
    pages = 3 * B * H * most + 50
    lens, table, shares, free = _state(rng, B, H, most, pages)
    parent = rng.integers(-1, B, B)
    keep = rng.integers(-5, 64 * most, B) if cut else None
    _check_fork(rng, parent, keep, lens, table, shares, free, pages, 64 if H < 100 else 128, in_place)


@pytest.mark.parametrize("D", [64, 128])
def test_one_prompt_many_forks(D):
    rng = np.random.default_rng(D)
    for B, n in ((64, 5000), (130, 64), (2, 1), (1030, 65), (3, 0)):
        most = -(-max(n, 1) // 64)
        lens, table = np.zeros(B, dtype=np.int64), np.full((B, 2, most), -1)
        pages = 2 * most + 2 * B + 9
        order = list(rng.permutation(pages))
        lens[B // 2] = n
        for j in range(-(-n // 64)):
            table[B // 2, :, j] = order.pop(), order.pop()
        s = _check_fork(rng, np.full(B, B // 2), None, lens, table, np.zeros(pages), order, pages, D)
        assert (s["seq_len"] == n).all()


@pytest.mark.parametrize("case", ["stay", "end", "swap", "few_pages", "no_pages", "bad_parents", "bad_lengths", "bad_pages",
                                  "bad_free", "keep_zero", "keep_all", "negative_keep", "held_elsewhere", "rollback"])
@pytest.mark.parametrize("in_place", [False, True])
def test_fork_bounds(case, in_place):
    rng = np.random.default_rng(11)
    B, H, most, pages = 40, 2, 6, 900
    lens, table, shares, free = _state(rng, B, H, most, pages, 4)
    parent, keep = rng.integers(-1, B, B), None
    if case == "stay":
        parent = np.arange(B)
    elif case == "end":
        parent[:] = -1
    elif case == "swap":
        parent = rng.permutation(B)
    elif case == "few_pages":
        free = free[:11]
        parent[:] = 3
    elif case == "no_pages":
        free = []
        parent[:] = rng.integers(0, 4, B)
    elif case == "bad_parents":
        parent[::3] = rng.choice([B, -2, 2**31 - 1, -2**31], len(parent[::3]))
    elif case == "bad_lengths":
        lens[[1, 5, 9]] = -1, 64 * most + 1, 2**31 - 1
        parent[[0, 1, 2, 3]] = 1, 1, 5, 9
    elif case == "bad_pages":
        table[4, 0, 0], table[4, 1, 1], table[7] = pages, -2**31, 2**31 - 1
        parent[[1, 4, 6, 7]] = 4, 4, 7, 7
    elif case == "bad_free":
        free[-9::2] = [pages, -1, -2**31, 2**31 - 1, pages + 5]
        parent[:] = rng.integers(0, 4, B)
    elif case == "keep_zero":
        keep = np.zeros(B)
    elif case == "keep_all":
        keep = np.full(B, 2**31 - 1)
    elif case == "negative_keep":
        keep = np.full(B, -2**31)
        keep[::2] = 70
    elif case == "held_elsewhere":   # a page that someone outside the table holds as well is copied
        shares[table[3, :, (lens[3] - 1) // 64]] += 1
        parent[[2, 3]] = 3, -1
    elif case == "rollback":
        parent, keep = np.arange(B), np.maximum(lens - rng.integers(0, 9, B), 0)
    if case in ("bad_lengths", "bad_pages", "bad_free"):   # what no step leaves: counts may only fall short, never below
        shares = shares + 1000
    _check_fork(rng, parent, keep, lens, table, shares, free, pages, 64, in_place)


def test_fork_then_assign_then_end():
    """A prompt, its forks, their own tokens, and every page back at the end."""
    rng = np.random.default_rng(5)
    B, H, most, pages = 6, 2, 8, 150
    c = ca.Cache(B, H, H, 64, most, pages)
    d = _devs(np.zeros(B), np.full((B, H, most), -1), np.zeros(pages), list(range(pages)), pages)
    pools = _pools(rng, pages, 64)
    d["free_count"].fill_(pages)
    d["free_pages"].copy_(torch.arange(pages, device=DEV))
    state = dict(seq_len=d["seq_len"], free_count=d["free_count"])

    def add(new):
        a = ca.assign_slots(c, i32_dev(new), int(sum(new)), d["seq_len"], d["page_table"], d["free_pages"],
                            d["free_count"], dict(state))
        return a["slot_map"]

    add([200] + [0] * 5)
    ca.sharing.fork_requests(c, i32_dev([0] * B), *[d[n] for n in NAMES], pools, bufs=dict(d))
    slots = [add([1] * B) for _ in range(70)]
    every = torch.stack(slots).flatten().tolist()
    assert min(every) >= 0 and len(set(every)) == len(every)     # no two write to one place
    assert d["seq_len"].tolist() == [270] * B
    assert int(d["free_count"]) == pages - (3 + 2 * B) * H       # three pages of the prompt are shared
    ca.sharing.fork_requests(c, i32_dev([-1] * B), *[d[n] for n in NAMES], pools, bufs=dict(d))
    assert int(d["free_count"]) == pages and sorted(d["free_pages"].tolist()) == list(range(pages))
    assert d["seq_len"].tolist() == [0] * B and not d["page_shares"].any()


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,H,most,pages,shared,D", [
    (1, 1, 2, 5, True, 64), (6, 2, 9, 300, True, 64), (20, 8, 5, 2000, True, 128), (3, 2, 4, 70000, False, 64),
    (64, 1, 12, 1100, False, 128), (2, 1, 1, 2, True, 64),
])
def test_compact(B, H, most, pages, shared, D, in_place):
    rng = np.random.default_rng(pages)
    lens, table, shares, free = _state(rng, B, H, most, pages, 3 if pages > 5 else 1, 60)
    for kind in ("as_is", "all_free", "none_free", "odd_list"):
        if kind == "all_free":
            lens_, free_ = np.zeros(B), list(rng.permutation(pages))
        elif kind == "none_free":
            lens_, free_ = lens, []
        else:
            lens_, free_ = lens, list(free)
        if kind == "odd_list" and free_:
            free_ = (free_ + [free_[0], pages, -1, -2**31, 2**31 - 1])[-pages:]
        want = sharing.compact_pages(lens_, table, shares if shared else None, free_, pages)
        c = ca.Cache(B, H, H, D, most, pages)
        pools = _pools(rng, pages, D)
        before = [p.clone() for p in pools]
        d = _devs(lens_, table, shares, free_, pages)
        if not shared:
            d["page_shares"] = None
        names = [n for n in NAMES if n != "seq_len"]
        bufs = {n: d[n] for n in names if d[n] is not None} if in_place else {}
        ws = torch.full((ca.sharing.compact_workspace_bytes(c),), 0xff, dtype=torch.uint8, device=DEV)
        got = ca.sharing.compact_pages(c, d["seq_len"], *[d[n] for n in names], pools, bufs=bufs, ws=ws)
        torch.cuda.synchronize()
        assert np.array_equal(got["new_page"].cpu().numpy(), want["new_page"])
        live = np.broadcast_to(np.arange(most) < -(-np.asarray(lens_, dtype=int) // 64)[:, None, None], table.shape)
        assert np.array_equal(got["page_table"].cpu().numpy()[live], want["page_table"][live])
        if shared:
            assert np.array_equal(got["page_shares"].cpu().numpy(), want["page_shares"])
        else:
            assert got.get("page_shares") is None
        n = len(want["free"])
        assert int(got["free_count"]) == n and got["free_pages"].tolist()[:n] == want["free"]
        for p, b in zip(pools, before):
            old = b.clone()
            for x, y in want["moved"].items():
                b[y] = old[x]
            assert torch.equal(p.view(torch.int16), b.view(torch.int16))


def test_calls_in_a_graph_and_on_a_stream():
    """Captured forks and compactions, replayed on other contents, equal the eager calls."""
    rng = np.random.default_rng(2)
    B, H, most, pages = 24, 2, 5, 700
    c = ca.Cache(B, H, H, 64, most, pages)
    states = [_state(rng, B, H, most, pages, 3) for _ in range(3)]
    parents = [rng.integers(-1, B, B) for _ in range(3)]
    pools = _pools(rng, pages, 64)
    d = _devs(*states[0], pages)
    parent, after = i32_dev(parents[0]), {n: torch.full_like(d[n], -3) for n in NAMES}
    ws, ws2 = (torch.zeros(f(c), dtype=torch.uint8, device=DEV)
               for f in (ca.sharing.fork_workspace_bytes, ca.sharing.compact_workspace_bytes))
    packed = {n: torch.full_like(d[n], -3) for n in NAMES if n != "seq_len"}
    packed["new_page"] = torch.full((pages,), -3, dtype=torch.int32, device=DEV)

    def step(stream=None):
        ca.sharing.fork_requests(c, parent, *[d[n] for n in NAMES], pools, bufs=after, ws=ws, stream=stream)
        ca.sharing.compact_pages(c, *[after[n] for n in NAMES], pools, bufs=packed, ws=ws2, stream=stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for s, par in list(zip(states, parents)) * 2:
        for n, t in _devs(*s, pages).items():
            d[n].copy_(t)
        parent.copy_(i32_dev(par))
        ws.fill_(0x77)
        g.replay()
        torch.cuda.synchronize()
        f = sharing.fork_requests(par, None, *s[:3], s[3], pages)
        p = sharing.compact_pages(f["seq_len"], f["page_table"], f["page_shares"], f["free"], pages)
        assert np.array_equal(after["page_shares"].cpu().numpy(), f["page_shares"])
        live = np.broadcast_to(np.arange(most) < -(-f["seq_len"] // 64)[:, None, None], (B, H, most))
        assert np.array_equal(packed["page_table"].cpu().numpy()[live], p["page_table"][live])
        assert int(packed["free_count"]) == len(p["free"])


@pytest.mark.parametrize("in_place", [False, True])
def test_more_rows_than_lds_holds(in_place):
    """Marks of more than 4096 rows are in the workspace, and forks of one row are counted in several rounds."""
    rng = np.random.default_rng(17)
    B, most = 4200, 2
    pages = 2 * B * most + 50
    lens, table, shares, free = _state(rng, B, 1, most, pages, 2, 100)
    parent = np.where(rng.random(B) < 0.6, 4150, rng.integers(-1, B, B))
    lens[4150] = max(lens[4150], 1)
    if table[4150, 0, 0] < 0:
        table[4150, 0, 0] = free.pop()
    _check_fork(rng, parent, rng.integers(0, 129, B), lens, table, shares, free, pages, 64, in_place)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("pages", [31, 32, 33, 1024, 8160, 16351, 16383, 16384, 16385])
def test_compact_of_small_and_larger_pools(pages, in_place):
    """Sizes at which the last word of a map in LDS ends, and on both sides of the largest pool with one."""
    test_compact(4, 2 if pages > 40 else 1, 2 if pages < 40 else 20, pages, True, 64, in_place)


@pytest.mark.parametrize("in_place", [False, True])
def test_counts_below_zero_write_nothing_out_of_range(in_place):
    """A count of -1 in one chunk of the ids takes a page off the places of the next chunk's: with no free page
    before, its first would be listed at -1.  Every output lies between guards."""
    rng = np.random.default_rng(21)
    B, most, pages = 8, 2, 700
    c = ca.Cache(B, 1, 1, 64, most, pages)
    pools = _pools(rng, pages, 64)
    shapes = dict(seq_len=(B,), page_table=(B, 1, most), page_shares=(pages,), free_pages=(pages,), free_count=(1,))
    for case in range(20):
        lens = np.array([64, 0, 64, 0, 128, 100, 0, 64])
        table, shares = np.full((B, 1, most), -1), np.zeros(pages, dtype=np.int64)
        table[0, 0, 0], table[2, 0, 0], table[4, 0], table[5, 0], table[7, 0, 0] = 3, 300, (10, 520), (11, 521), 690
        parent = np.array([0, 0, -1, 3, 4, 4, 0, -1])
        shares[3] = -1
        if case:
            shares = rng.integers(-3, 2, pages)
            parent = rng.integers(-1, B, B)
        free = [] if case % 2 == 0 else [600, 601]
        guarded = {n: torch.full((int(np.prod(s)) + 128,), -77, dtype=torch.int32, device=DEV) for n, s in shapes.items()}
        bufs = {n: guarded[n][64:64 + int(np.prod(s))].view(s) for n, s in shapes.items()}
        d = _devs(lens, table, shares, free, pages)
        if in_place:
            for n in NAMES:
                bufs[n].copy_(d[n])
            d = dict(bufs)
        ca.sharing.fork_requests(c, i32_dev(parent), *[d[n] for n in NAMES], pools, bufs=bufs)
        torch.cuda.synchronize()
        for n, t in guarded.items():
            assert (t[:64] == -77).all() and (t[-64:] == -77).all(), (case, n)
        assert 0 <= int(bufs["free_count"]) <= pages
