"""Decode attention where a wave has many pages: hundreds of them, from a small pool whose
pages the page table lists over and over.

Tolerances.  lse = (m + log2 sum) ln 2 with m the scaled maximum.  Of m: half a step for the
constant log2 e, for the sum with log2, for ln 2 and for the product, 2^-24 each of |lse|.  Of
the sum: half a step for every page that a wave adds and for each of the 16 adds within a page, two
steps for the exponential, and 8 for the joins.  A weight's factor for an earlier maximum that
stays is 1, so nothing else grows with the pages.
"""
import numpy as np
import pytest
import torch

import synth
from _helpers import bf16_dev, bf16_host_f64, i32_dev
from oracle import serving

pytestmark = pytest.mark.gpu

ca = pytest.importorskip("paper_2605_16839_amd")
DEV = "cuda"
BF16_HALF = 2.0 ** -8
WAVES = 256 * 8


def _roundings():
    """Whole scores up to 256 whose product with log2 e fp32 rounds up most, and down most."""
    n = np.arange(180, 257)
    c = np.float32(1.4426950408889634)
    off = (n.astype(np.float32) * c).astype(np.float64) - n * np.float64(c)
    return [int(n[off.argmax()]), int(n[off.argmin()])]


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("top", _roundings())
def test_a_maximum_that_stays(top, layout):
    """The same largest scores in every page: no page weighs more for being read earlier."""
    rng = np.random.default_rng(top)
    B, Hq, Hkv, D, cycle, times = 64, 8, 4, 64, 7, 585
    blocks = cycle * times
    pages = B * Hkv * blocks / WAVES
    below = rng.integers(0, 6, (cycle, 64))
    below[:, 0] = 0
    k = np.zeros((cycle, 64, D), dtype=np.float32)
    k[..., 3] = top - below                       # exact in bf16, and so are the scores
    v = synth.bf16_round(rng.standard_normal((cycle, 64, D)).astype(np.float32))
    q = np.zeros((B, Hq, D), dtype=np.float32)
    q[..., 3] = 1
    kp, q = synth.bf16_round(k), synth.bf16_round(q)
    table = np.broadcast_to(np.arange(blocks) % cycle, (B, Hkv, blocks))
    c = ca.Cache(B, Hq, Hkv, D, blocks, cycle, v_layout=layout)
    lse = torch.empty(B, Hq, device=DEV)
    vd = v if layout == 0 else synth.v_pages_transposed(v)
    out, _ = ca.decode_attention(c, bf16_dev(q), (bf16_dev(kp), bf16_dev(vd)), i32_dev(table),
                                 i32_dev([blocks * 64] * B), 1.0, lse=lse)
    ref, one, mass, _ = serving.decode_attention(q[:1], kp, v, table[:1, :, :cycle], [cycle * 64], 1.0)
    want = one[0] + np.log(times)
    tol = 4 * 2.0 ** -24 * np.abs(want) + (pages + 16 + 4 + 8) * 2.0 ** -24
    off = np.abs(lse.cpu().numpy().astype(np.float64) - want)
    assert (off <= tol).all(), (off.max(), tol.max())
    # values: two sums with as many roundings, weights of 16 bits
    tol = BF16_HALF * np.abs(ref) + (2.0 ** -16 + 4 * (pages + 28) * 2.0 ** -24) * mass
    assert (np.abs(bf16_host_f64(out) - ref) <= tol).all()


def _check(rng, lens, Hq, Hkv, D, layout, most, pool, sample, tables=None, gs=0):
    """Every request's pages are drawn from a small pool; a sample of requests against the oracle,
    all rows against a second call."""
    B = len(lens)
    kp, vp = (synth.bf16_round(rng.standard_normal((pool, 64, D)).astype(np.float32)) for _ in "kv")
    q = synth.bf16_round(rng.standard_normal((B, Hq, D)).astype(np.float32))
    table = rng.integers(0, pool, (B, Hkv, most))
    c = ca.Cache(B, Hq, Hkv, D, most, pool, v_layout=layout)
    lse = torch.empty(B, Hq, device=DEV)
    csr = None
    if tables:
        rows = [r for t in tables for r in t]
        ip = np.concatenate([[0], np.cumsum([len(r) for r in rows])])
        ix = np.zeros(len(rows) * most)
        ix[:ip[-1]] = [j for r in rows for j in r]
        csr = (i32_dev(ip), i32_dev(ix))
    args = (c, bf16_dev(q), (bf16_dev(kp), bf16_dev(vp if layout == 0 else synth.v_pages_transposed(vp))),
            i32_dev(table), i32_dev(lens), D ** -0.5)
    out, _ = ca.decode_attention(*args, lse=lse, tables=csr, group_size=gs)
    again, _ = ca.decode_attention(*args, tables=csr, group_size=gs)
    assert torch.equal(out, again)
    sample = list(sample)
    ref, ref_lse, mass, size = serving.decode_attention(q[sample], kp, vp, table[sample], [lens[b] for b in sample],
                                                        D ** -0.5, [tables[b] for b in sample] if tables else None, gs)
    got, gl = bf16_host_f64(out)[sample], lse.cpu().numpy().astype(np.float64)[sample]
    pages = sum(-(-n // 64) for n in lens) * Hkv / WAVES + 1
    delta = D * 2.0 ** -23 * size
    steps = (pages + 28) * 2.0 ** -24
    tol = BF16_HALF * np.abs(ref) + (2.0 ** -16 + 2 * delta[..., None] + 4 * steps) * mass
    assert (np.abs(got - ref) <= tol).all(), np.argwhere(np.abs(got - ref) > tol)[:5].tolist()
    fin = np.isfinite(ref_lse)
    assert np.array_equal(gl[~fin], ref_lse[~fin])
    off = np.abs(gl[fin] - ref_lse[fin])
    assert (off <= delta[fin] + 4 * 2.0 ** -24 * np.abs(ref_lse[fin]) + steps).all()


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("Hq,Hkv,D", [(8, 8, 64), (16, 4, 128), (12, 1, 64), (18, 2, 128)])
def test_more_than_64_pages_to_a_wave(Hq, Hkv, D, layout):
    """Page ids are fetched 64 at a time: rows of about as many, and of many more, in shares of
    more than 128 pages that they begin, end and cross."""
    rng = np.random.default_rng(Hq)
    blocks = [63, 64, 65, 1, 127, 128, 129, 2, 191, 192, 193, 700, 62, 66, 1023]
    B = 2600 // Hkv
    take = rng.integers(0, len(blocks), B)
    lens = [64 * blocks[i] - int(rng.integers(0, 64)) for i in take]
    lens[0], lens[B - 1], lens[7] = 64 * 1024, 64 * 65, 0
    assert sum(-(-n // 64) for n in lens) * Hkv > 128 * WAVES
    sample = sorted({0, 7, B - 1, *rng.choice(B, 8, replace=False).tolist()})
    _check(rng, lens, Hq, Hkv, D, layout, 1024, 300, sample)


def test_more_than_64_pages_to_a_wave_of_few_requests():
    """One lane to a request."""
    rng = np.random.default_rng(3)
    lens = [64 * int(n) - 5 for n in rng.integers(500, 4000, 40)]
    for layout in (0, 1):
        _check(rng, lens, 8, 4, 64, layout, 4096, 200, [0, 11, 39])


def test_more_than_64_listed_pages_to_a_wave():
    rng = np.random.default_rng(4)
    B, Hq, Hkv, gs, most = 128, 16, 8, 1, 512
    lens = [64 * most - 7] * B
    some = [sorted(rng.choice(most, int(n), replace=False).tolist()) for n in (63, 64, 65, 129, 200, 511, 512, 0)]
    tables = [[some[int(i)] for i in rng.integers(0, len(some), Hq // gs)] for _ in range(B)]
    tables[5][3] = some[6]
    assert sum(len(r) for t in tables for r in t) > 96 * WAVES
    for layout in (0, 1):
        _check(rng, lens, Hq, Hkv, 64, layout, most, 200, [0, 5, 77, 127], tables, gs)


@pytest.mark.parametrize("gap", [1, 62, 63, 64, 65, 127, 128, 1000])
def test_idle_requests_inside_a_share(gap):
    """A wave goes from one request to the next over those that have nothing."""
    rng = np.random.default_rng(gap)
    lens = [64 * 401 + 5] + [0] * gap + [64 * 200] + [0] * gap + [64 * 399 - 1, 3] + [0] * gap
    live = [0, gap + 1, 2 * gap + 2, 2 * gap + 3]
    sample = [0, 1, gap, gap + 1, gap + 2, *live[2:], len(lens) - 1]
    _check(rng, lens, 16, 8, 64, gap % 2, 402, 500, sample)
    # over tables: rows of no block between rows of some
    B, Hq, gs = 3, 256, 1
    rows = [[list(range(90))] + [[]] * (Hq - 2) + [list(range(7, 96))] for _ in range(B)]
    _check(rng, [64 * 96] * B, Hq, 4, 64, gap % 2, 96, 300, range(B), rows, gs)


def test_idle_requests_inside_a_share_cost_little():
    """4000 idle requests between two live ones, three times: one load after the other for each of them
    took 16 times the batch without them; 64 at a time take 3 times."""
    Hq, Hkv, D, pool = 16, 8, 64, 500
    live = [64 * 401 + 5, 64 * 200, 64 * 399 - 1, 3]
    took = []
    for gap in (70, 4000):     # without a gap there are 70 idle ones behind
        lens = live + [0] * gap if gap == 70 else [x for n in live[:3] for x in [n] + [0] * gap] + [3]
        B = len(lens)
        c = ca.Cache(B, Hq, Hkv, D, 402, pool)
        pools = tuple(torch.zeros(pool, 64, D, dtype=torch.bfloat16, device=DEV) for _ in "kv")
        q = torch.zeros(B, Hq, D, dtype=torch.bfloat16, device=DEV)
        table, kl = torch.zeros(B, Hkv, 402, dtype=torch.int32, device=DEV), i32_dev(lens)
        out, ws = torch.empty_like(q), torch.zeros(ca.decode_workspace_bytes(c), dtype=torch.uint8, device=DEV)
        best = float("inf")
        for _ in range(20):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in "ab")
            a.record()
            for _ in range(10):
                ca.decode_attention(c, q, pools, table, kl, 0.125, out=out, ws=ws)
            b.record()
            torch.cuda.synchronize()
            best = min(best, a.elapsed_time(b))
        took.append(best)
    assert took[1] < 8 * took[0], took
