"""The serving step's kernels against the float64 oracle: pages and slots exactly, the rotary
append and the decode attention within what their roundings allow.

Tolerances.  A stored bf16 is off by at most 2^-8 of its value.
  rotary: the turn is exact to half an fp32 step of at most half a turn (2^-25 turns =
    2^-22.3 rad), cosine and sine to a few steps (2^-22), the two products and their sum to
    3 * 2^-24: together below 2^-20 * (|a| + |b|) before the store.
  attention: a score sums D exact products in fp32, off by at most
    delta = D * 2^-23 * max_j sm_scale sum_d |q_d k_jd|; a weight by 2 delta and 2^-20 for
    the exponential; with more than 8 heads on a KV head the weights are bf16 (2^-8), with
    fewer their rest is kept (2^-16).  All of it scales sum_j w_j |v_j|.
"""
import math

import numpy as np
import pytest
import torch

import oracle
import synth
from _helpers import bf16_dev, bf16_host_f64, i32_dev
from oracle import serving

pytestmark = pytest.mark.gpu

ca = pytest.importorskip("paper_2605_16839_amd")
DEV = "cuda"
BF16_HALF = 2.0 ** -8


def _bf16(rng, shape, scale=1.0):
    return synth.bf16_round((rng.standard_normal(shape) * scale).astype(np.float32))


# ---------------------------------------------------------------------------
# pages and slots
# ---------------------------------------------------------------------------
def _requests(rng, B, Hkv, max_blocks, longest, spare):
    lens = rng.integers(0, longest + 1, B)
    lens[rng.random(B) < 0.2] = 0
    blocks = -(-lens // 64)
    pages = int(blocks.sum()) * Hkv + spare
    order = list(rng.permutation(pages))
    table = np.full((B, Hkv, max_blocks), -7)
    for b in range(B):
        for j in range(blocks[b]):
            for h in range(Hkv):
                table[b, h, j] = order.pop()
    return lens, table, order, pages


def _free_dev(free, capacity):
    a = np.full(max(capacity, 1), -3)
    a[:len(free)] = free
    return i32_dev(a[:capacity])


def _check_assign(B, Hkv, max_blocks, lens, new, table, free, pages, T, in_place=False, capacity=None):
    want = serving.assign_slots(new, T, lens, table, free, pages)
    c = ca.Cache(B, Hkv, Hkv, 64, max_blocks, pages)
    seq, count, pt = i32_dev(lens), i32_dev([len(free)]), i32_dev(table)
    fp = _free_dev(free, capacity or len(free) + 1)
    bufs = {True: dict(seq_len=seq, free_count=count), "len": dict(seq_len=seq),
            "count": dict(free_count=count)}.get(in_place, {})
    got = ca.assign_slots(c, i32_dev(new), T, seq, pt, fp, count, bufs)
    torch.cuda.synchronize()
    for key in ("slot_map", "positions", "token_indptr", "granted", "seq_len", "free_count"):
        assert np.array_equal(got[key].cpu().numpy(), want[key]), key
    assert np.array_equal(pt.cpu().numpy(), want["page_table"])
    assert np.array_equal(fp.cpu().numpy()[:len(free)], free)        # only read
    if not in_place:
        assert np.array_equal(seq.cpu().numpy(), lens) and int(count) == len(free)


@pytest.mark.parametrize("in_place", [False, True, "len", "count"])
@pytest.mark.parametrize("B,Hkv,longest,most_new,pad", [
    (1, 1, 0, 1, 0), (1, 8, 700, 2048, 0), (3, 2, 64, 130, 5), (64, 8, 3000, 2, 0),
    (255, 1, 500, 3, 1), (256, 4, 100, 70, 0), (257, 2, 100, 70, 300), (1000, 3, 900, 2, 4),
    (5, 8, 5000, 3000, 1500), (2, 1500, 70, 70, 3), (2049, 1, 64, 2, 0),
])
def test_assign_slots(B, Hkv, longest, most_new, pad, in_place):
    rng = np.random.default_rng(B * 31 + Hkv)
    max_blocks = -(-(longest + most_new) // 64)
    new = rng.integers(0, most_new + 1, B)
    lens, table, free, pages = _requests(rng, B, Hkv, max_blocks, longest, B * Hkv * (most_new // 64 + 2))
    _check_assign(B, Hkv, max_blocks, lens, new, table, free, pages, int(new.sum()) + pad, in_place)


@pytest.mark.parametrize("case", ["no_tokens", "no_pages", "few_pages", "rows_end", "too_long",
                                  "bad_lengths", "bad_pages", "bad_free_pages", "huge_new", "no_list"])
def test_assign_slots_bounds(case):
    rng = np.random.default_rng(5)
    B, Hkv, max_blocks = 300, 2, 6
    lens, table, free, pages = _requests(rng, B, Hkv, max_blocks, 250, 900)
    new = rng.integers(0, 90, B)
    T = int(new.sum())
    if case == "no_tokens":
        new[:] = 0
        T = 0
    elif case == "no_pages":
        free = []
    elif case == "few_pages":
        free = free[:101]
    elif case == "rows_end":
        T //= 2
    elif case == "too_long":
        new[::7] = 64 * max_blocks + 1 - lens[::7]
        T = int(new.sum()) - 3
    elif case == "bad_lengths":
        lens[3], lens[40], new[77], new[299] = -1, 64 * max_blocks + 5, -2, -2**31
        lens[41] = 2**31 - 1
        T = int(np.maximum(new, 0).sum())
    elif case == "bad_pages":
        table[10:60] = pages
        table[60:90] = -2**31
        lens[10:90] |= 1      # their last block is held
    elif case == "bad_free_pages":    # they are given away, but nothing is written to them
        free[-40::3] = [pages, -1, -2**31, 2**31 - 1] * 3 + [pages + 1] * 2
    elif case == "huge_new":
        new[100:] = 2**31 - 1   # the row sum passes 32 bits
    elif case == "no_list":
        free = []
        new = np.minimum(new, -lens % 64)
        T = int(new.sum())
    _check_assign(B, Hkv, max_blocks, lens, new, table, free, pages, T, capacity=0 if case == "no_list" else None)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,Hkv,longest,share,short", [
    (1, 1, 64, 1.0, 0), (1, 8, 100000, 1.0, 0), (100, 8, 3000, 0.1, 0), (300, 2, 500, 0.6, 100),
    (513, 1, 100, 1.0, 0), (40, 4, 900, 0.0, 0),
])
def test_release_pages(B, Hkv, longest, share, short, in_place):
    rng = np.random.default_rng(B + Hkv)
    max_blocks = -(-longest // 64) + 1
    lens, table, free, pages = _requests(rng, B, Hkv, max_blocks, longest, 50)
    if B == 1:
        lens[:] = longest
        table[0] = rng.permutation(Hkv * max_blocks).reshape(Hkv, max_blocks)
        pages = Hkv * max_blocks + 50
        free = list(range(pages - 50, pages))
    release = (rng.random(B) < share).astype(np.int64) * rng.integers(1, 9, B)
    if B > 200:
        lens[7], lens[200], release[7], release[200] = -1, 64 * max_blocks + 1, 1, 1
    capacity = pages - short
    want_len, want = serving.release_pages(release, lens, table, free, capacity, max_blocks)
    c = ca.Cache(B, Hkv, Hkv, 64, max_blocks, pages)
    seq, count, pt, fp = i32_dev(lens), i32_dev([len(free)]), i32_dev(table), _free_dev(free, capacity)
    got = ca.release_pages(c, i32_dev(release), seq, pt, fp, count,
                           out=(seq, count) if in_place else None)
    torch.cuda.synchronize()
    assert got[0].cpu().tolist() == want_len and int(got[1]) == len(want)
    assert fp.cpu().tolist()[:len(want)] == want
    assert (fp.cpu().numpy()[len(want):] == -3).all()         # rows behind are left alone


# ---------------------------------------------------------------------------
# rotary append
# ---------------------------------------------------------------------------
def _append_case(rng, T, Hq, Hkv, D, layout, rot, axes, interleaved, strided, skip=0.1, far=131072,
                 ordered=False):
    pages = max(2, -(-T * Hkv // 64) + 3)
    slots = rng.permutation(pages * 64)[:T * Hkv].reshape(T, Hkv)
    if ordered:     # runs of consecutive slots, as a prompt's tokens have
        slots = np.stack([np.arange(T) + h * (-(-T // 64) + 1) * 64 + 5 for h in range(Hkv)], 1)
        pages = (Hkv + 1) * (-(-T // 64) + 2)
    slots = np.where(rng.random((T, Hkv)) < skip, rng.choice([-1, pages * 64, -2**40, 2**40], (T, Hkv)), slots)
    pos = rng.integers(0, far, (axes, T))
    f = (500000.0 ** (-np.arange(rot // 2) / max(rot // 2, 1))).astype(np.float32)
    pair_axis = rng.integers(0, axes, rot // 2).tolist() if axes > 1 else None
    qkv = _bf16(rng, (T, Hq + 2 * Hkv, D))
    kp, vp = _bf16(rng, (pages, 64, D)), _bf16(rng, (pages, 64, D))
    c = ca.Cache(1, Hq, Hkv, D, 1, pages, v_layout=layout)
    r = ca.Rotary(torch.from_numpy(f).to(DEV) if rot else None, interleaved, axes, pair_axis)
    t = bf16_dev(qkv)
    parts = [t[:, :Hq], t[:, Hq:Hq + Hkv], t[:, Hq + Hkv:]]
    if not strided:
        parts = [x.contiguous() for x in parts]
    vd = vp if layout == ca.V_TOKEN_MAJOR else synth.v_pages_transposed(vp)
    pools = (bf16_dev(kp), bf16_dev(vd))
    positions = i32_dev(pos if axes > 1 else pos[0])
    q = ca.rotary_append(c, r, *parts, positions, torch.from_numpy(slots).to(DEV), pools)
    torch.cuda.synchronize()

    x = oracle.bf16_to_f64(qkv)
    turned = serving.rotate(x[:, :Hq + Hkv], pos, f, pair_axis, interleaved)
    both = np.abs(x[:, :Hq + Hkv])
    pair = both.copy()            # |a| + |b| of every element's pair, 0 where nothing turns
    n = rot // 2
    if interleaved:
        s = both[..., 0:rot:2] + both[..., 1:rot:2]
        pair[..., 0:rot:2], pair[..., 1:rot:2] = s, s
    else:
        s = both[..., :n] + both[..., n:rot]
        pair[..., :n], pair[..., n:rot] = s, s
    tol = BF16_HALF * np.abs(turned) + 2.0 ** -20 * pair
    tol[..., rot:] = 0            # copied as they are
    got = bf16_host_f64(q)
    assert (np.abs(got - turned[:, :Hq]) <= tol[:, :Hq]).all()
    want, allow = oracle.bf16_to_f64(kp), np.zeros((pages, 64, D))
    vwant = vp.copy()
    for i in range(T):
        for h in range(Hkv):
            s = int(slots[i, h])
            if 0 <= s < pages * 64:
                want[s // 64, s % 64] = turned[i, Hq + h]
                allow[s // 64, s % 64] = tol[i, Hq + h]
                vwant[s // 64, s % 64] = qkv[i, Hq + Hkv + h]
    assert (np.abs(bf16_host_f64(pools[0]) - want) <= allow).all()      # other rows bit for bit
    if layout != ca.V_TOKEN_MAJOR:
        vwant = synth.v_pages_transposed(vwant)
    assert np.array_equal(pools[1].view(torch.int16).cpu().numpy().view(np.uint16), vwant)


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("T,Hq,Hkv,D,rot,axes,interleaved,strided", [
    (1, 4, 1, 64, 64, 1, False, True), (1, 32, 8, 128, 128, 1, False, False),
    (64, 32, 8, 128, 128, 3, False, True), (3, 9, 9, 64, 32, 1, True, True),
    (257, 28, 4, 128, 128, 4, True, False), (130, 16, 1, 128, 96, 2, False, True),
    (1000, 8, 2, 64, 16, 1, False, True), (70, 5, 5, 128, 0, 1, False, True),
    (65, 71, 1, 64, 48, 1, True, True),
])
def test_rotary_append(T, Hq, Hkv, D, rot, axes, interleaved, strided, layout):
    _append_case(np.random.default_rng(T + Hq), T, Hq, Hkv, D, layout, rot, axes, interleaved, strided)


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("T,Hkv,D", [(7, 2, 64), (200, 2, 128), (1451, 1, 128), (2048, 4, 64)])
def test_rotary_append_runs(T, Hkv, D, layout):
    """Consecutive slots that start inside a page, whole or with holes."""
    for skip in (0.0, 0.02):
        _append_case(np.random.default_rng(T), T, 2 * Hkv, Hkv, D, layout, D, 1, False, True, skip,
                     ordered=True)


def test_rotary_far_positions():
    _append_case(np.random.default_rng(3), 40, 4, 2, 128, 0, 128, 2, False, True, far=2**31 - 1)
    # negative places (an axis may count from a centre)
    rng = np.random.default_rng(4)
    c = ca.Cache(1, 2, 2, 64, 1, 2)
    f = (100.0 ** (-np.arange(32) / 32)).astype(np.float32)
    x = _bf16(rng, (5, 2, 64))
    pos = -rng.integers(0, 10**6, 5)
    q = ca.rotary_append(c, ca.Rotary(torch.from_numpy(f).to(DEV)), bf16_dev(x), bf16_dev(x), bf16_dev(x),
                         i32_dev(pos), torch.full((5, 2), -1, device=DEV),
                         tuple(torch.zeros(2, 64, 64, device=DEV, dtype=torch.bfloat16) for _ in "kv"))
    y = oracle.bf16_to_f64(x)
    want = serving.rotate(y, pos[None], f)
    pair = np.concatenate([np.abs(y[..., :32]) + np.abs(y[..., 32:])] * 2, -1)
    assert (np.abs(bf16_host_f64(q) - want) <= BF16_HALF * np.abs(want) + 2.0 ** -20 * pair).all()


def test_rotary_append_in_place_and_empty():
    rng = np.random.default_rng(8)
    c = ca.Cache(1, 8, 2, 128, 1, 9)
    f = torch.from_numpy((1e4 ** (-np.arange(64) / 64)).astype(np.float32)).to(DEV)
    q, k, v = (bf16_dev(_bf16(rng, (300, h, 128))) for h in (8, 2, 2))
    pools = tuple(bf16_dev(_bf16(rng, (9, 64, 128))) for _ in "kv")
    pos, slots = i32_dev(rng.integers(0, 999, 300)), torch.full((300, 2), -1, device=DEV)
    want = ca.rotary_append(c, ca.Rotary(f), q, k, v, pos, slots, pools)
    before = [x.clone() for x in pools]
    same = ca.rotary_append(c, ca.Rotary(f), q, k, v, pos, slots, pools, out=q)
    assert same is q and torch.equal(q, want)
    assert all(torch.equal(a, b) for a, b in zip(before, pools))
    none = ca.rotary_append(c, ca.Rotary(f), q[:0], k[:0], v[:0], pos[:0], slots[:0], pools)
    assert none.shape == (0, 8, 128)


def test_binding_refuses():
    c = ca.Cache(2, 4, 2, 64, 3, 9)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)  # noqa: E731
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device=DEV)  # noqa: E731
    pools, slots = (bf(9, 64, 64), bf(9, 64, 64)), torch.zeros(5, 2, dtype=torch.int64, device=DEV)
    r = ca.Rotary(torch.ones(32, device=DEV))
    for q, k, pos, sl, kv in [(bf(5, 4, 64).float(), bf(5, 2, 64), i32(5), slots, pools),
                              (bf(5, 4, 64), bf(4, 2, 64), i32(5), slots, pools),
                              (bf(5, 4, 64), bf(5, 64, 2).transpose(1, 2), i32(5), slots, pools),
                              (bf(5, 4, 64), bf(5, 2, 64), i32(4), slots, pools),
                              (bf(5, 4, 64), bf(5, 2, 64), i32(3, 5), slots, pools),
                              (bf(5, 4, 64), bf(5, 2, 64), i32(5), slots.int(), pools),
                              (bf(5, 4, 64), bf(5, 2, 64), i32(5), slots, (pools[0], bf(9, 64, 128)))]:
        with pytest.raises(ValueError):
            ca.rotary_append(c, r, q, k, k, pos, sl, kv)
    for q, kl, table, kw in [(bf(2, 4, 64), i32(3), i32(2, 2, 3), {}),
                             (bf(2, 4, 64), i32(2), i32(2, 2, 4), {}),
                             (bf(2, 4, 64), i32(2).long(), i32(2, 2, 3), {}),
                             (bf(2, 4, 64), i32(2), i32(2, 2, 3), dict(tables=(i32(5), i32(11)))),
                             (bf(2, 4, 64), i32(2), i32(2, 2, 3), dict(lse=bf(2, 4)))]:
        with pytest.raises(ValueError):
            ca.decode_attention(c, q, pools, table, kl, 0.1, **kw)
    with pytest.raises(ValueError):
        ca.assign_slots(c, i32(2), 4, i32(2), i32(2, 2, 3), i32(5), i32(2))


# ---------------------------------------------------------------------------
# decode attention
# ---------------------------------------------------------------------------
def _pools(rng, lens, Hkv, D, max_blocks, poison=True):
    """Pools and a page table; NaN and infinities behind the last token, page ids that no one
    may follow behind the last block."""
    blocks = [-(-max(n, 0) // 64) for n in lens]
    pages = sum(blocks) * Hkv + 2
    order = list(rng.permutation(pages))
    table = rng.choice([-1, pages, 2**31 - 1, 0], (len(lens), Hkv, max_blocks))
    kp, vp = _bf16(rng, (pages, 64, D)), _bf16(rng, (pages, 64, D))
    for b, n in enumerate(lens):
        for j in range(blocks[b]):
            for h in range(Hkv):
                p = table[b, h, j] = order.pop()
                if poison and n - 64 * j < 64:
                    kp[p, n - 64 * j:] = rng.choice([0x7fc0, 0x7f80, 0xff80])
                    vp[p, n - 64 * j:] = rng.choice([0x7fc0, 0x7f80, 0xff80])
    return kp, vp, table, pages


def _csr(tables, max_blocks):
    rows = [r for t in tables for r in t]
    ip = np.concatenate([[0], np.cumsum([len(r) for r in rows])])
    ix = np.full(len(rows) * max_blocks, 2**30)
    ix[:ip[-1]] = [j for r in rows for j in r]
    return i32_dev(ip), i32_dev(ix)


def _attention_ok(out, lse, q, kp, vp, table, lens, scale, tables=None, gs=0, heads_per_kv=1):
    ref, ref_lse, mass, size = serving.decode_attention(q, kp, vp, table, lens, scale, tables, gs)
    D = q.shape[-1]
    delta = D * 2.0 ** -23 * size[..., None]
    weight = 2.0 ** -16 if heads_per_kv <= 8 else BF16_HALF
    got = bf16_host_f64(out)
    assert np.isfinite(got).all()
    err, tol = np.abs(got - ref), BF16_HALF * np.abs(ref) + (weight + 2 * delta + 2.0 ** -20) * mass
    assert (err <= tol).all(), (np.max(err - tol), np.argwhere(err > tol)[:5])
    gl = lse.cpu().numpy().astype(np.float64)
    assert np.array_equal(np.isfinite(gl), np.isfinite(ref_lse))
    assert (gl[~np.isfinite(ref_lse)] == -np.inf).all()
    fin = np.isfinite(ref_lse)
    d, size = np.abs(gl[fin] - ref_lse[fin]), np.maximum(1, np.abs(ref_lse[fin]))
    assert (d <= delta[..., 0][fin] + 2.0 ** -20 * size).all()


def _run_decode(rng, lens, Hq, Hkv, D, layout, max_blocks=None, gs=0, tables=None, scale=None, qscale=2.0):
    max_blocks = max_blocks or max(1, max(-(-n // 64) for n in lens))
    kp, vp, table, pages = _pools(rng, lens, Hkv, D, max_blocks)
    q = _bf16(rng, (len(lens), Hq, D), qscale)
    scale = scale or D ** -0.5
    c = ca.Cache(len(lens), Hq, Hkv, D, max_blocks, pages, v_layout=layout)
    vd = vp if layout == ca.V_TOKEN_MAJOR else synth.v_pages_transposed(vp)
    lse = torch.full((len(lens), Hq), 7.0, device=DEV)
    out = torch.full((len(lens), Hq, D), 9.0, device=DEV, dtype=torch.bfloat16)
    # a workspace of no particular contents
    ws = torch.full((max(ca.decode_workspace_bytes(c, gs), 16),), 0xff, dtype=torch.uint8, device=DEV)
    args = (c, bf16_dev(q), (bf16_dev(kp), bf16_dev(vd)), i32_dev(table), i32_dev(lens), scale)
    kw = dict(tables=_csr(tables, max_blocks) if tables else None, group_size=gs, ws=ws)
    ca.decode_attention(*args, out=out, lse=lse, **kw)
    torch.cuda.synchronize()
    _attention_ok(out, lse, q, kp, vp, table, lens, scale, tables, gs, Hq // Hkv)
    for _ in range(2):      # the same bits again, without lse too
        again, _ = ca.decode_attention(*args, **kw)
        assert torch.equal(again, out)


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("Hq,Hkv,D", [(4, 1, 64), (32, 8, 128), (8, 8, 64), (28, 4, 128), (9, 1, 128),
                                      (16, 1, 64), (20, 1, 128), (40, 1, 64), (71, 1, 64), (8, 1, 128)])
def test_decode_attention(Hq, Hkv, D, layout):
    rng = np.random.default_rng(Hq * 7 + D)
    _run_decode(rng, [1, 0, 63, 64, 65, 700, 0, 129, 2048], Hq, Hkv, D, layout)


@pytest.mark.parametrize("lens,Hkv,max_blocks", [
    ([0], 1, 1), ([1], 1, 1), ([1], 8, 2048), ([64], 2, 1), ([0, 0, 0], 4, 5), ([5000], 1, None),
    ([20001, 3], 2, 16384), ([12345, 1, 0, 4097, 640], 8, 300), ([128] * 40, 8, None),
    ([3, 1] * 150, 2, None), ([65] * 700, 1, None), ([0] * 1030 + [200, 0, 77], 1, 9),
])
def test_decode_lengths(lens, Hkv, max_blocks):
    rng = np.random.default_rng(len(lens) + Hkv)
    for layout in (0, 1):
        _run_decode(rng, lens, 2 * Hkv, Hkv, 64 if len(lens) > 100 else 128, layout, max_blocks)


@pytest.mark.parametrize("Hq,Hkv,D,lens,max_blocks", [
    # more than 8 rows: the last workgroup of a row joins it, of many pieces here
    (4, 1, 128, [20001] + [0] * 8, None), (16, 1, 128, [0] * 9 + [17000], None),
    (9, 3, 64, [9000, 0, 8191, 1], None), (71, 1, 64, [5000, 70], None),
    # 8 rows at most and long tables: a launch of its own joins them
    (4, 1, 128, [30000], 600), (40, 1, 64, [9000], 200), (16, 8, 128, [12000], 2048),
    (20, 2, 128, [5000, 9001], 300), (1, 1, 64, [16000], 250), (8, 1, 64, [0, 7000, 64], 129),
])
def test_decode_rows_of_many_pieces(Hq, Hkv, D, lens, max_blocks):
    rng = np.random.default_rng(Hq + len(lens))
    for layout in (0, 1):
        _run_decode(rng, lens, Hq, Hkv, D, layout, max_blocks)


@pytest.mark.parametrize("lens,Hkv,max_blocks", [
    # on both sides of a page to a workgroup (128 pages), of two (512), of whole rows (4 pages on average)
    ([64 * 64], 1, 64), ([64 * 128], 1, 129), ([64 * 128 + 1], 1, 129), ([64 * 64], 2, 64),
    ([64 * 511 + 9], 1, 512), ([64 * 512], 1, 512), ([64 * 513], 1, 513),
    ([256], 8, 4), ([257], 8, 5), ([192, 130, 1], 8, None), ([900, 1, 1, 60], 2, None),
    ([300, 1, 64, 0, 190, 256, 512, 1], 16, None), ([256] * 32, 8, None), ([256] * 31 + [257], 8, None),
    ([3000] + [64] * 60, 4, None), ([64] * 255 + [4000], 1, None),
])
def test_decode_few_pages(lens, Hkv, max_blocks):
    rng = np.random.default_rng(sum(lens) + Hkv)
    for layout in (0, 1):
        _run_decode(rng, lens, 4 * Hkv, Hkv, 64, layout, max_blocks)


@pytest.mark.parametrize("B", [64, 65, 4096, 4097, 5000])
def test_decode_many_requests(B):
    """A lane sums several requests, 64 and more of them at last."""
    rng = np.random.default_rng(B)
    lens = np.where(rng.random(B) < 0.7, 0, rng.integers(1, 140, B))
    lens[[0, B - 1]] = 100, 65
    _run_decode(rng, lens.tolist(), 2, 1, 64, 0)
    if B == 4097:
        _run_decode(rng, [0] * (B - 1) + [1], 2, 1, 64, 0)
        _run_decode(rng, [300] + [0] * (B - 1), 2, 1, 64, 1)


def test_decode_more_rows_than_workgroups():
    rng = np.random.default_rng(0)
    _run_decode(rng, rng.integers(0, 200, 700).tolist(), 8, 8, 64, 0)
    _run_decode(rng, rng.integers(0, 2000, 90).tolist(), 16, 4, 64, 1)


@pytest.mark.parametrize("scale,qscale", [(1.0, 1.0), (4.0, 3.0), (1e-3, 1.0)])
def test_decode_sharp_and_flat(scale, qscale):
    _run_decode(np.random.default_rng(1), [3000, 77], 8, 2, 128, 0, scale=scale, qscale=qscale)


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("Hq,Hkv,gs", [(32, 8, 4), (32, 4, 4), (32, 4, 8), (28, 4, 7), (28, 4, 1), (40, 1, 20)])
def test_decode_tables(Hq, Hkv, gs, layout):
    rng = np.random.default_rng(Hq + gs)
    lens = [1, 0, 64, 5000, 1000, 130]
    tables = []
    for n in lens:
        blocks = -(-n // 64)
        tables.append([sorted(rng.choice(blocks, rng.integers(0, blocks + 1), replace=False).tolist())
                       for _ in range(Hq // gs)])
    tables[3][0] = list(range(79))
    tables[4][-1] = []
    _run_decode(rng, lens, Hq, Hkv, 128, layout, gs=gs, tables=tables)


@pytest.mark.parametrize("Hq,Hkv,gs,lens,max_blocks", [(8, 2, 4, [20000], 400), (8, 2, 2, [9000, 0], 200),
                                                       (40, 1, 20, [9000], 150), (8, 1, 1, [12000], 188)])
def test_decode_long_tables(Hq, Hkv, gs, lens, max_blocks):
    rng = np.random.default_rng(gs)
    tables = [[sorted(rng.choice(-(-n // 64), -(-n // 80), replace=False).tolist()) if n else []
               for _ in range(Hq // gs)] for n in lens]
    for layout in (0, 1):
        _run_decode(rng, lens, Hq, Hkv, 128, layout, max_blocks, gs, tables)


def test_decode_out_of_range_is_never_followed():
    """Lengths, page ids, table entries and row bounds that are out of range."""
    rng = np.random.default_rng(6)
    lens, Hq, Hkv, D, most = [300, 200, 150, 64, 100], 4, 2, 64, 6
    kp, vp, table, pages = _pools(rng, lens, Hkv, D, most, poison=False)
    q = _bf16(rng, (5, Hq, D))
    c = ca.Cache(5, Hq, Hkv, D, most, pages)
    dev = (bf16_dev(q), (bf16_dev(kp), bf16_dev(vp)))
    lse = torch.empty(5, Hq, device=DEV)
    # page ids: the block's keys are left out
    bad = table.copy()
    bad[0, 0, 1], bad[0, 1, 0], bad[2, :, :], bad[4, :, 1] = pages, -1, 2**31 - 1, -2**31
    without = [[[0, 2, 3, 4], [1, 2, 3, 4]], [[0, 1, 2, 3]] * 2, [[], []], [[0]] * 2, [[0]] * 2]
    out, _ = ca.decode_attention(c, *dev, i32_dev(bad), i32_dev(lens), 0.125, lse=lse)
    _attention_ok(out, lse, q, kp, vp, table, lens, 0.125, without)
    # lengths: 0 below 0, the table's end above it
    full = rng.integers(0, pages, (5, Hkv, most))
    out, _ = ca.decode_attention(c, *dev, i32_dev(full), i32_dev([-1, -2**31, 64 * most + 1, 2**31 - 1, 5]),
                                 0.125, lse=lse)
    _attention_ok(out, lse, q, kp, vp, full, [0, 0, 64 * most, 64 * most, 5], 0.125)
    # table entries: left out; the entry of a block past the length too
    T = [[[0, 1, 4], [2]], [[-1, 0, 9], [4]], [[1, 2**31 - 1], [0]], [[0], [-2**31]], [[0, 1], [1]]]
    kept = [[[j for j in r if 0 <= j < -(-n // 64)] for r in t] for n, t in zip(lens, T)]
    out, _ = ca.decode_attention(c, *dev, i32_dev(table), i32_dev(lens), 0.125, tables=_csr(T, most), lse=lse)
    _attention_ok(out, lse, q, kp, vp, table, lens, 0.125, kept)
    # row bounds that descend, are negative or pass the capacity: whatever they give, it ends
    ip, ix = _csr(kept, most)
    for at, v in [(3, 2**31 - 1), (0, -5), (10, 2**30), (5, 0), (1, -2**31)]:
        worse = ip.clone()
        worse[at] = v
        ca.decode_attention(c, *dev, i32_dev(table), i32_dev(lens), 0.125, tables=(worse, ix), lse=lse)
    torch.cuda.synchronize()


def test_decode_not_finite():
    rng = np.random.default_rng(7)
    lens, Hq, Hkv, D = [500, 40, 64], 6, 2, 64
    kp, vp, table, pages = _pools(rng, lens, Hkv, D, 8)
    q = _bf16(rng, (3, Hq, D))
    kp[table[0, 0, 3], 5, 2] = 0x7fc0                  # NaN: heads 0..2 of request 0
    q[1, 4], kp[table[1, 1, 0], 7] = 0x3f80, 0x7f80    # +inf score: head 4 of request 1
    q[2, 1], kp[table[2, 0, 0], 9] = 0x3f80, 0xff80    # -inf score: the key has no weight
    q[1, 3], q[1, 5], q[2, 0], q[2, 2] = 0xbf80, 0xbf80, 0x3f80, 0x3f80   # -inf, -inf; as head 1
    c = ca.Cache(3, Hq, Hkv, D, 8, pages)
    lse = torch.empty(3, Hq, device=DEV)
    out, _ = ca.decode_attention(c, bf16_dev(q), (bf16_dev(kp), bf16_dev(vp)), i32_dev(table), i32_dev(lens),
                                 0.125, lse=lse)
    got, gl = bf16_host_f64(out), lse.cpu().numpy()
    gone = np.zeros((3, Hq), dtype=bool)
    gone[0, :3] = gone[1, 4] = True
    assert np.isnan(got[gone]).all() and (gl[gone] == -np.inf).all()
    assert np.isfinite(got[~gone]).all() and np.isfinite(gl[~gone]).all()
    # every score -inf: no key is seen
    kp[table[2, 1, 0]] = 0x7f80
    q[2, 3:] = 0xbf80
    out, _ = ca.decode_attention(c, bf16_dev(q), (bf16_dev(kp), bf16_dev(vp)), i32_dev(table), i32_dev(lens),
                                 0.125, lse=lse)
    assert (out[2, 3:] == 0).all() and (lse[2, 3:] == -math.inf).all()


def test_decode_far_pages():
    """Pages whose elements lie past 2^32."""
    rng = np.random.default_rng(9)
    D, pages = 128, 600000
    kp, vp = (torch.empty(pages, 64, D, dtype=torch.bfloat16, device=DEV) for _ in "kv")
    ids = np.array([[[599999, 3, 524289], [262145, 599998, 0]]])
    small = [_bf16(rng, (6, 64, D)) for _ in "kv"]
    for pool, s in zip((kp, vp), small):
        pool[torch.from_numpy(ids.ravel()).to(DEV)] = bf16_dev(s)
    q = _bf16(rng, (1, 4, D))
    lse = torch.empty(1, 4, device=DEV)
    for layout in (0, 1):
        if layout:
            for i in ids.ravel():
                vp[i] = vp[i].t().reshape(64, D)
        c = ca.Cache(1, 4, 2, D, 3, pages, v_layout=layout)
        pool = vp if layout == 0 else vp.view(pages, D, 64)
        out, _ = ca.decode_attention(c, bf16_dev(q), (kp, pool), i32_dev(ids), i32_dev([170]), 0.09, lse=lse)
        _attention_ok(out, lse, q, *small, np.arange(6).reshape(1, 2, 3), [170], 0.09)


# ---------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------
class _Server:
    """The serving loop's buffers; the host mirrors requests only to check the results."""

    def __init__(self, rng, B, Hq, Hkv, D, most, pages, layout):
        self.rng, self.D, self.scale = rng, D, D ** -0.5
        self.c = ca.Cache(B, Hq, Hkv, D, most, pages, v_layout=layout)
        self.pools = tuple(torch.zeros(s, dtype=torch.bfloat16, device=DEV)
                           for s in ((pages, 64, D), (pages, 64, D) if layout == 0 else (pages, D, 64)))
        self.table = torch.full((B, Hkv, most), -1, dtype=torch.int32, device=DEV)
        self.free = i32_dev(rng.permutation(pages))
        self.state = dict(seq_len=i32_dev([0] * B), free_count=i32_dev([pages]))
        self.freq = torch.from_numpy((1e4 ** (-np.arange(D // 2) / (D // 2))).astype(np.float32)).to(DEV)
        self.rot = ca.Rotary(self.freq)
        self.ws = torch.zeros(max(ca.decode_workspace_bytes(self.c), 16), dtype=torch.uint8, device=DEV)
        self.rope = {}                                      # (request, position) -> rotated k, v

    def step(self, new, qkv, T, bufs=None):
        Hq, Hkv = self.c.num_q_heads, self.c.num_kv_heads
        b = ca.assign_slots(self.c, new, T, self.state["seq_len"], self.table, self.free,
                            self.state["free_count"], {**(bufs or {}), **self.state})
        q = ca.rotary_append(self.c, self.rot, qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:],
                             b["positions"], b["slot_map"], self.pools)
        return b, q

    def remember(self, new, lens, qkv):
        """The host's copy of what the step appended, from the inputs alone."""
        Hq, Hkv = self.c.num_q_heads, self.c.num_kv_heads
        x = oracle.bf16_to_f64(qkv)
        row = 0
        for b, n in enumerate(new):
            for i in range(n):
                p = int(lens[b]) + i
                k = serving.rotate(x[row:row + 1, Hq:Hq + Hkv], np.array([[p]]), self.freq.cpu().numpy())
                self.rope[b, p] = (k[0], x[row, Hq + Hkv:])
                row += 1

    def expected(self, qkv_row, b, n):
        """Decode attention of request b with n cached tokens (the last is its own)."""
        Hq, Hkv = self.c.num_q_heads, self.c.num_kv_heads
        q = serving.rotate(oracle.bf16_to_f64(qkv_row)[None, :Hq], np.array([[n - 1]]), self.freq.cpu().numpy())[0]
        k = np.stack([self.rope[b, p][0] for p in range(n)], 1)      # [Hkv, n, D]
        v = np.stack([self.rope[b, p][1] for p in range(n)], 1)
        out = np.zeros((Hq, self.D))
        for h in range(Hq):
            x = self.scale * k[h // (Hq // Hkv)] @ q[h]
            w = np.exp(x - x.max())
            out[h] = w @ v[h // (Hq // Hkv)] / w.sum()
        return out


@pytest.mark.parametrize("layout", [0, 1])
def test_serving_steps_together(layout):
    """Prompts in ragged chunks, decode steps, a request that ends and one that takes its place,
    the prompt chunk read by the dense chunk attention.  bf16 roundings of q, k and the weights
    enter the scores: the comparison is loose (2e-2), the bookkeeping is exact."""
    rng = np.random.default_rng(10 + layout)
    B, Hq, Hkv, D, most, pages = 4, 8, 2, 64, 6, 40
    s = _Server(rng, B, Hq, Hkv, D, most, pages, layout)
    lens = [0] * B
    for new, ended in [([70, 0, 130, 5], []), ([1, 40, 1, 1], []), ([1, 1, 1, 1], [2]), ([1, 1, 200, 1], []),
                       ([1, 1, 1, 1], [0, 3]), ([64, 1, 1, 1], []), ([1, 1, 1, 1], [])]:
        for b in ended:
            lens[b] = 0
        if ended:
            flags = [int(b in ended) for b in range(B)]
            ca.release_pages(s.c, i32_dev(flags), s.state["seq_len"], s.table, s.free, s.state["free_count"],
                             out=(s.state["seq_len"], s.state["free_count"]))
        T = sum(new) + 3
        qkv = _bf16(rng, (T, Hq + 2 * Hkv, D))
        b, q = s.step(i32_dev(new), bf16_dev(qkv), T)
        s.remember(new, lens, qkv)
        lens = [x + n for x, n in zip(lens, new)]
        assert b["granted"].cpu().tolist() == new and s.state["seq_len"].cpu().tolist() == lens
        held = sum(-(-n // 64) for n in lens) * Hkv
        assert int(s.state["free_count"]) == pages - held
        # one query per request: its last token's
        ends = b["token_indptr"].cpu().tolist()
        last = [e - 1 for e in ends[1:]]
        out, _ = ca.decode_attention(s.c, q[torch.tensor(last, device=DEV)].contiguous(), s.pools, s.table,
                                     s.state["seq_len"], s.scale, ws=s.ws)
        got = bf16_host_f64(out)
        for i in range(B):
            if new[i] and lens[i]:
                want = s.expected(qkv[last[i]], i, lens[i])
                assert np.abs(got[i] - want).max() <= 2e-2, (i, lens[i])
        # the same tokens through the chunk path: a chunk of one token per request
        if all(new):
            p = ca.Problem(B, Hq, Hkv, D, 64, 1, most, [n - 1 for n in lens], v_layout=layout)
            chunk, _ = ca.dense_paged_chunk_attention(p, q[torch.tensor(last, device=DEV)][:, None].contiguous(),
                                                      s.pools, s.table, s.scale)
            assert np.abs(got - bf16_host_f64(chunk)[:, 0]).max() <= 2e-2


def test_prefill_chunk_through_the_new_cache():
    """assign_slots and rotary_append fill the cache that the selector, the tables and the chunk
    attention then read; decode_attention over those tables and over all blocks follows."""
    rng = np.random.default_rng(12)
    B, Hq, Hkv, D, C, most = 2, 8, 2, 128, 200, 12
    s = _Server(rng, B, Hq, Hkv, D, most, 60, 0)
    lens = [0, 0]
    for _ in range(3):
        qkv = _bf16(rng, (B * C, Hq + 2 * Hkv, D))
        _, q = s.step(i32_dev([C] * B), bf16_dev(qkv), B * C)
        lens = [n + C for n in lens]
        p = ca.Problem(B, Hq, Hkv, D, 64, C, most, [n - C for n in lens])
        tables, _ = ca.estimate_tables(p, q.view(B, C, Hq, D), s.pools[0], s.table, 1.0, 4)
        sel, _ = ca.chunk_attention(p, q.view(B, C, Hq, D), s.pools, s.table, tables, 4, s.scale)
        dense, _ = ca.dense_paged_chunk_attention(p, q.view(B, C, Hq, D), s.pools, s.table, s.scale)
        assert (sel.float() - dense.float()).abs().max() <= 2e-2      # top_frac 1: every block
        last = q.view(B, C, Hq, D)[:, -1].contiguous()
        out, _ = ca.decode_attention(s.c, last, s.pools, s.table, s.state["seq_len"], s.scale)
        assert (out.float() - dense[:, -1].float()).abs().max() <= 2e-2
        some, _ = ca.decode_attention(s.c, last, s.pools, s.table, s.state["seq_len"], s.scale, tables=tables,
                                      group_size=4)
        assert (some.float() - sel[:, -1].float()).abs().max() <= 2e-2


def test_captured_step_replays_while_requests_grow():
    """A decode step captured once: each replay sees the lengths the last one left, pages open
    while it is replayed, and equals the same step run eagerly on a copy of the state."""
    rng = np.random.default_rng(11)
    B, Hq, Hkv, D, most, pages = 5, 8, 2, 128, 5, 60
    a, e = (_Server(np.random.default_rng(1), B, Hq, Hkv, D, most, pages, 0) for _ in range(2))
    prompt = _bf16(rng, (250, Hq + 2 * Hkv, D))
    first = i32_dev([62, 0, 100, 1, 63])
    for s in (a, e):
        s.step(first, bf16_dev(prompt), 250)
    new, qkv = i32_dev([1, 0, 1, 1, 1]), bf16_dev(_bf16(rng, (B, Hq + 2 * Hkv, D)))
    lse = {id(s): torch.empty(B, Hq, device=DEV) for s in (a, e)}

    def step(s):
        b, q = s.step(new, qkv, B)
        out, _ = ca.decode_attention(s.c, q, s.pools, s.table, s.state["seq_len"], s.scale, lse=lse[id(s)],
                                     ws=s.ws)
        return b, out

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    keep = {k: v.clone() for k, v in a.state.items()}
    with torch.cuda.stream(side):
        step(a)                                   # a first call outside the capture
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for k, v in keep.items():                     # undo it: its pages are dealt again
        a.state[k].copy_(v)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b, out = step(a)
    for i in range(9):
        qkv.copy_(bf16_dev(_bf16(rng, (B, Hq + 2 * Hkv, D))))
        eb, eout = step(e)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(b["slot_map"], eb["slot_map"]), i
        assert torch.equal(out, eout) and torch.equal(lse[id(a)], lse[id(e)])
        assert torch.equal(a.state["seq_len"], e.state["seq_len"])
        assert torch.equal(a.table, e.table) and torch.equal(a.pools[0], e.pools[0])


def test_streams_by_argument():
    """stream= takes each call to that stream: after work there that the current stream lacks."""
    rng = np.random.default_rng(15)
    B, Hq, Hkv, D, most, pages = 3, 4, 2, 64, 4, 30
    a, e = (_Server(np.random.default_rng(2), B, Hq, Hkv, D, most, pages, 0) for _ in range(2))
    qkv, new = bf16_dev(_bf16(rng, (B, Hq + 2 * Hkv, D))), i32_dev([1, 1, 1])
    eb, eq = e.step(new, qkv, B)
    eout, _ = ca.decode_attention(e.c, eq, e.pools, e.table, e.state["seq_len"], e.scale)
    elen, ecount = ca.release_pages(e.c, i32_dev([0, 1, 0]), e.state["seq_len"], e.table, e.free, e.state["free_count"])
    st = torch.cuda.Stream()
    late, q, out = torch.zeros_like(qkv), torch.empty(B, Hq, D, dtype=qkv.dtype, device=DEV), torch.empty_like(eout)
    bufs = {**{k: torch.zeros_like(v) for k, v in eb.items()}, **a.state}
    flags, ended = i32_dev([0, 1, 0]), (torch.empty_like(elen), torch.empty_like(ecount))
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        torch.cuda._sleep(20_000_000)
        late.copy_(qkv)
    ca.assign_slots(a.c, new, B, a.state["seq_len"], a.table, a.free, a.state["free_count"], bufs, stream=st)
    ca.rotary_append(a.c, a.rot, late[:, :Hq], late[:, Hq:Hq + Hkv], late[:, Hq + Hkv:], bufs["positions"],
                     bufs["slot_map"], a.pools, out=q, stream=st)
    ca.decode_attention(a.c, q, a.pools, a.table, a.state["seq_len"], a.scale, out=out, ws=a.ws, stream=st)
    ca.release_pages(a.c, flags, a.state["seq_len"], a.table, a.free, a.state["free_count"], out=ended, stream=st)
    st.synchronize()
    assert torch.equal(q, eq) and torch.equal(out, eout) and torch.equal(a.pools[0], e.pools[0])
    assert torch.equal(ended[0], elen) and torch.equal(ended[1], ecount) and torch.equal(a.free, e.free)


def test_another_stream_and_two_workspaces():
    rng = np.random.default_rng(13)
    lens, Hq, Hkv, D = [4000, 100], 8, 2, 64
    kp, vp, table, pages = _pools(rng, lens, Hkv, D, 70)
    c = ca.Cache(2, Hq, Hkv, D, 70, pages)
    q = [bf16_dev(_bf16(rng, (2, Hq, D))) for _ in range(2)]
    pools, pt, kl = (bf16_dev(kp), bf16_dev(vp)), i32_dev(table), i32_dev(lens)
    want = [ca.decode_attention(c, x, pools, pt, kl, 0.125)[0] for x in q]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for x, st in zip(q, streams):
            with torch.cuda.stream(st):
                got.append(ca.decode_attention(c, x, pools, pt, kl, 0.125)[0])
    torch.cuda.synchronize()
    for i, x in enumerate(got):
        assert torch.equal(x, want[i % 2])


def test_one_workspace_for_several_sizes_and_graphs():
    """Calls of other sizes, eager and captured, leave a workspace that the next can use."""
    rng = np.random.default_rng(14)
    cases = []
    for lens, Hq, Hkv, D, most in [([7000, 3000], 32, 8, 128, 110), ([500] * 20, 8, 2, 64, 9),
                                   ([3000, 0, 64], 16, 4, 64, 47), ([12000], 4, 1, 128, 200)]:
        kp, vp, table, pages = _pools(rng, lens, Hkv, D, most)
        c = ca.Cache(len(lens), Hq, Hkv, D, most, pages)
        args = (c, bf16_dev(_bf16(rng, (len(lens), Hq, D))), (bf16_dev(kp), bf16_dev(vp)), i32_dev(table),
                i32_dev(lens), 0.1)
        cases.append((args, ca.decode_attention(*args)[0]))
    ws = torch.full((max(ca.decode_workspace_bytes(a[0]) for a, _ in cases),), 0xff, dtype=torch.uint8, device=DEV)
    for _ in range(3):
        for args, want in cases:
            assert torch.equal(ca.decode_attention(*args, ws=ws)[0], want)
    torch.cuda.synchronize()
    graphs = []
    for args, want in (cases[0], cases[1], cases[3]):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out, _ = ca.decode_attention(*args, ws=ws)
        graphs.append((g, out, want))
    for i in range(4):
        for g, out, want in graphs:
            out.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want), i
        args, want = cases[2 + i % 2]
        assert torch.equal(ca.decode_attention(*args, ws=ws)[0], want)
