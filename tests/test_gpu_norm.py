"""The rotary append with norms of the heads against the oracle.

Tolerance.  A square, and a sum of D = 64 or 128 of them over 16 in a lane and 8 lanes, is off by at most
(1 + 16 + 3) * 2^-24 of the sum (all terms are positive); the mean, eps, the square root (1 ulp), its
reciprocal (1 ulp) and the products with weight and value add at most 8 * 2^-24, and half of the sum's error
counts under the root: together below 2^-19 of each normalised element.  The weight with its offset rounds
once, 2^-24 of (1 + |w|).  The turn adds 2^-20 * (|a| + |b|) (the turn itself is exact to 2^-22.3), the store
2^-8 of the value at most; a subnormal or tiny result counts 2^-133.
"""
import numpy as np
import pytest
import torch

import oracle
import synth
from _helpers import bf16_dev, bf16_host_f64, i32_dev
from oracle import serving, sharing

pytestmark = pytest.mark.gpu

ca = pytest.importorskip("paper_2605_16839_amd")
DEV = "cuda"
BF16_HALF = 2.0 ** -8


def _bf16(rng, shape, scale=1.0):
    return synth.bf16_round((rng.standard_normal(shape) * scale).astype(np.float32))


def _weight(rng, D, wide, offset):
    """On the GPU, and as it counts."""
    w = (1 + 0.3 * rng.standard_normal(D) - offset).astype(np.float32)
    if wide:
        return torch.from_numpy(w).to(DEV), w.astype(np.float64) + offset
    bits = synth.bf16_round(w)
    return bf16_dev(bits), oracle.bf16_to_f64(bits) + offset


def _case(rng, T, Hq, Hkv, D, layout=0, rot=None, axes=1, interleaved=False, wide=False, offset=0, eps=1e-6,
          sides="qk", scale=1.0, strided=True, x=None):
    rot = D if rot is None else rot
    pages = max(2, -(-T * Hkv // 64) + 3)
    slots = rng.permutation(pages * 64)[:T * Hkv].reshape(T, Hkv)
    slots = np.where(rng.random((T, Hkv)) < 0.1, rng.choice([-1, pages * 64, -2**40, 2**40], (T, Hkv)), slots)
    pos = rng.integers(0, 131072, (axes, T))
    f = (500000.0 ** (-np.arange(rot // 2) / max(rot // 2, 1))).astype(np.float32)
    pair_axis = rng.integers(0, axes, rot // 2).tolist() if axes > 1 else None
    qkv = _bf16(rng, (T, Hq + 2 * Hkv, D), scale) if x is None else x
    kp, vp = _bf16(rng, (pages, 64, D)), _bf16(rng, (pages, 64, D))
    qw, qv = _weight(rng, D, wide, offset) if "q" in sides else (None, None)
    kw, kv = _weight(rng, D, wide, offset) if "k" in sides else (None, None)
    c = ca.Cache(1, Hq, Hkv, D, 1, pages, v_layout=layout)
    r = ca.Rotary(torch.from_numpy(f).to(DEV) if rot else None, interleaved, axes, pair_axis,
                  norm=ca.HeadNorm(qw, kw, eps=eps, unit_offset=bool(offset)))
    t = bf16_dev(qkv)
    parts = [t[:, :Hq], t[:, Hq:Hq + Hkv], t[:, Hq + Hkv:]]
    if not strided:
        parts = [p.contiguous() for p in parts]
    pools = (bf16_dev(kp), bf16_dev(vp if layout == 0 else synth.v_pages_transposed(vp)))
    positions, slot_map = i32_dev(pos if axes > 1 else pos[0]), torch.from_numpy(slots).to(DEV)
    q = ca.rotary_append(c, r, *parts, positions, slot_map, pools)
    torch.cuda.synchronize()

    y = oracle.bf16_to_f64(qkv)
    heads = np.concatenate([sharing.normed(y[:, :Hq], qv, eps), sharing.normed(y[:, Hq:Hq + Hkv], kv, eps)], 1)
    want = serving.rotate(heads, pos, f, pair_axis, interleaved)
    each = np.abs(heads) * 2.0 ** -19          # of the norm
    for at, w in ((slice(0, Hq), qv), (slice(Hq, Hq + Hkv), kv)):
        if w is None:
            each[:, at] = 0
        elif offset:
            # the weight's rounding, of the element's share without the weight
            z = sharing.normed(y[:, at], np.ones(D), eps)
            each[:, at] += np.abs(z) * 2.0 ** -24 * (1 + np.abs(w))
    both, pair = np.abs(heads) * 2.0 ** -20 + each, np.abs(heads) * 0 + each
    n = rot // 2
    for a, b in ([(slice(0, rot, 2), slice(1, rot, 2))] if interleaved else [(slice(0, n), slice(n, rot))]):
        s = both[..., a] + both[..., b]
        pair[..., a], pair[..., b] = s, s
    tol = BF16_HALF * np.abs(want) + pair + 2.0 ** -133
    for at, w in ((slice(0, Hq), qv), (slice(Hq, Hq + Hkv), kv)):
        if w is None:
            tol[:, at, rot:] = 0               # copied as they are
    got = bf16_host_f64(q)
    assert (np.abs(got - want[:, :Hq]) <= tol[:, :Hq]).all()
    pool, allow, vwant = oracle.bf16_to_f64(kp), np.zeros((pages, 64, D)), vp.copy()
    for i in range(T):
        for h in range(Hkv):
            s = int(slots[i, h])
            if 0 <= s < pages * 64:
                pool[s // 64, s % 64], allow[s // 64, s % 64] = want[i, Hq + h], tol[i, Hq + h]
                vwant[s // 64, s % 64] = qkv[i, Hq + Hkv + h]
    assert (np.abs(bf16_host_f64(pools[0]) - pool) <= allow).all()       # other rows bit for bit
    vwant = vwant if layout == 0 else synth.v_pages_transposed(vwant)
    assert np.array_equal(pools[1].view(torch.int16).cpu().numpy().view(np.uint16), vwant)
    return q


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("T,Hq,Hkv,D,rot,axes,interleaved,wide,offset,strided", [
    (1, 4, 1, 64, 64, 1, False, False, 0, True), (1, 32, 8, 128, 128, 1, False, True, 1, False),
    (64, 32, 8, 128, 128, 3, False, False, 1, True), (3, 9, 9, 64, 32, 1, True, True, 0, True),
    (257, 28, 4, 128, 128, 4, True, True, 0, False), (130, 16, 1, 128, 96, 2, False, False, 0, True),
    (1000, 8, 2, 64, 16, 1, False, False, 1, True), (70, 5, 5, 128, 0, 1, False, True, 1, True),
    (65, 71, 1, 64, 48, 1, True, False, 0, True), (600, 4, 1, 128, 64, 1, False, False, 0, True),
])
def test_norm_rotary_append(T, Hq, Hkv, D, rot, axes, interleaved, wide, offset, strided, layout):
    _case(np.random.default_rng(T + Hq), T, Hq, Hkv, D, layout, rot, axes, interleaved, wide, offset, strided=strided)


@pytest.mark.parametrize("sides", ["q", "k", ""])
def test_one_side_only(sides):
    """The side without a weight is as it was without norms, bit for bit where nothing turns."""
    for rot in (128, 32):
        _case(np.random.default_rng(9), 33, 8, 2, 128, rot=rot, sides=sides)


@pytest.mark.parametrize("scale,eps", [(1e4, 0.0), (1e-3, 0.0), (1e-3, 1e-5), (1e-12, 1e-6), (1e17, 1e-6), (1.0, 1.0)])
def test_scales(scale, eps):
    _case(np.random.default_rng(10), 20, 4, 2, 128, scale=scale, eps=eps)
    _case(np.random.default_rng(11), 20, 4, 2, 64, scale=scale, eps=eps, wide=True, rot=0)


def test_heads_of_zeros_and_not_finite():
    rng = np.random.default_rng(12)
    x = _bf16(rng, (6, 8, 64))
    x[0] = 0                      # eps keeps them zeros
    _case(rng, 6, 4, 2, 64, x=x)
    c, T = ca.Cache(1, 4, 2, 64, 1, 2), 3
    one = torch.ones(64, device=DEV)
    t = bf16_dev(_bf16(rng, (T, 4, 64)))
    t[1, 2, 5], t[2, 0, 7] = float("nan"), float("inf")
    r = ca.Rotary(None, norm=ca.HeadNorm(one, one))
    k = t[:, :2].contiguous()
    q = ca.rotary_append(c, r, t, k, k, i32_dev(np.zeros(T)), torch.full((T, 2), -1, device=DEV),
                         tuple(torch.zeros(2, 64, 64, device=DEV, dtype=torch.bfloat16) for _ in "kv"))
    bad = q.isnan().any(-1)
    assert bad.nonzero().tolist() == [[1, 2], [2, 0]]             # other heads are not touched
    assert q[1, 2].isnan().all() and q[2, 0, 7].isnan() and not q[2, 0, :7].any()


def test_in_place_and_empty_and_refusals():
    rng = np.random.default_rng(8)
    c = ca.Cache(1, 8, 2, 128, 1, 9)
    w = torch.ones(128, device=DEV, dtype=torch.bfloat16)
    r = ca.Rotary(torch.ones(64, device=DEV), norm=ca.HeadNorm(w, w))
    q, k, v = (bf16_dev(_bf16(rng, (300, h, 128))) for h in (8, 2, 2))
    pools = tuple(bf16_dev(_bf16(rng, (9, 64, 128))) for _ in "kv")
    pos, slots = i32_dev(rng.integers(0, 999, 300)), torch.full((300, 2), -1, device=DEV)
    want = ca.rotary_append(c, r, q, k, v, pos, slots, pools)
    same = ca.rotary_append(c, r, q, k, v, pos, slots, pools, out=q)
    assert same is q and torch.equal(q, want)
    none = ca.rotary_append(c, r, q[:0], k[:0], v[:0], pos[:0], slots[:0], pools)
    assert none.shape == (0, 8, 128)
    for bad in (ca.HeadNorm(torch.ones(64, device=DEV), None), ca.HeadNorm(torch.ones(128), None)):
        with pytest.raises(ValueError, match="norm weights"):
            ca.rotary_append(c, ca.Rotary(None, norm=bad), q, k, v, pos, slots, pools)


def test_against_the_calls_apart():
    """Norm in 32 bits, then the plain rotary append of its bf16: one rounding more, so within 2^-7 or so."""
    rng = np.random.default_rng(3)
    T, Hq, Hkv, D = 50, 8, 2, 128
    c = ca.Cache(1, Hq, Hkv, D, 1, 9)
    f = torch.from_numpy((1e4 ** (-np.arange(64) / 64)).astype(np.float32)).to(DEV)
    q, k, v = (bf16_dev(_bf16(rng, (T, h, D))) for h in (Hq, Hkv, Hkv))
    w = bf16_dev(_bf16(rng, (D,)))
    pos, slots = i32_dev(rng.integers(0, 9999, T)), torch.arange(T * Hkv, device=DEV).view(T, Hkv)
    a, b = ([torch.zeros(9, 64, D, device=DEV, dtype=torch.bfloat16) for _ in "kv"] for _ in "ab")
    one = ca.rotary_append(c, ca.Rotary(f, norm=ca.HeadNorm(w, w, eps=1e-5)), q, k, v, pos, slots, tuple(a))
    n = [(x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-5) * w.float()).bfloat16() for x in (q, k)]
    two = ca.rotary_append(c, ca.Rotary(f), *n, v, pos, slots, tuple(b))
    # each of a pair's two elements is off by 2^-8 of it at most, and so the turned ones by that of their size
    size = lambda x: x.float().unflatten(-1, (2, 64)).norm(dim=-2).repeat(1, 1, 2)  # noqa: E731
    assert ((one.float() - two.float()).abs() <= size(n[0]) * (2 * BF16_HALF * 2 ** 0.5)).all()
    assert torch.equal(a[1], b[1]) and (a[0].float() - b[0].float()).norm() <= 2 * BF16_HALF * b[0].float().norm()


def test_graph_and_stream():
    rng = np.random.default_rng(4)
    T, c = 40, ca.Cache(1, 4, 2, 64, 1, 9)
    w = torch.ones(64, device=DEV)
    r = ca.Rotary(torch.ones(32, device=DEV), norm=ca.HeadNorm(w, w))
    q, k, v = (bf16_dev(_bf16(rng, (T, h, 64))) for h in (4, 2, 2))
    pools = tuple(torch.zeros(9, 64, 64, device=DEV, dtype=torch.bfloat16) for _ in "kv")
    pos, slots = i32_dev(np.arange(T)), torch.arange(2 * T, device=DEV).view(T, 2)
    out = torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ca.rotary_append(c, r, q, k, v, pos, slots, pools, out, side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ca.rotary_append(c, r, q, k, v, pos, slots, pools, out)
    for i in range(3):
        q.copy_(bf16_dev(_bf16(rng, (T, 4, 64))))
        w.fill_(1.0 + i)
        g.replay()
        torch.cuda.synchronize()
        got, kp = out.clone(), pools[0].clone()
        want = ca.rotary_append(c, r, q, k, v, pos, slots, pools)
        assert torch.equal(got, want) and torch.equal(kp, pools[0])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("power", [60, 61, 62, 63, 64, 100, 126, 127, -62, -63, -64, -75, -80, -100, -126, -130, -133])
def test_heads_of_any_size(D, power):
    """Squares and their sums stay in range wherever the elements are: mean squares on both sides of 2^121 and
    2^127, heads of the largest bf16 and of subnormal ones, with and without eps."""
    rng = np.random.default_rng(1000 + D + power)
    x = np.full((12, 8, D), np.float32(2.0) ** power)
    x[4:] *= rng.choice(np.float32([1, -1]), (8, 8, D))
    if power > -126:
        x[8:] *= rng.choice(np.float32([1, 2.0 ** -20, 2.0 ** -5]), (4, 8, D))
        x[8:, :, 5] = np.float32(2.0) ** power * np.float32(1.5)
    bits = synth.bf16_round(x)
    assert np.array_equal(synth.bf16_bits_to_f32(bits), x)
    for eps in (0.0, 1e-6, 1e-38):
        _case(rng, 12, 4, 2, D, x=bits, eps=eps)
    _case(rng, 12, 4, 2, D, x=bits, eps=0.0, wide=True, offset=1, rot=0)


@pytest.mark.parametrize("D", [64, 128])
def test_one_large_element(D):
    """A head whose largest element is far from the others, at the ends of what bf16 holds."""
    rng = np.random.default_rng(D)
    for large, small in ((3.3e38, 1e30), (1e20, 1e-20), (1e-20, 1e-38), (2.0 ** -100, 2.0 ** -133)):
        x = np.full((6, 8, D), np.float32(small))
        x[:, :, 7] = np.float32(large)
        for eps in (0.0, 1e-6):
            _case(rng, 6, 4, 2, D, x=synth.bf16_round(x), eps=eps)


@pytest.mark.parametrize("D", [64, 128])
def test_heads_of_all_sizes_side_by_side(D):
    """Scaled and unscaled heads in one wave, in any order."""
    rng = np.random.default_rng(40 + D)
    for Hq, Hkv in ((4, 2), (21, 7), (33, 1)):
        heads = Hq + 2 * Hkv
        x = rng.standard_normal((30, heads, D)).astype(np.float32)
        x *= np.float32(2.0) ** rng.choice([-120, -64, -20, -19, 0, 0, 0, 19, 21, 62, 120], (30, heads, 1)).astype(np.float32)
        _case(rng, 30, Hq, Hkv, D, x=synth.bf16_round(x), eps=0.0)
        _case(rng, 30, Hq, Hkv, D, x=synth.bf16_round(x), eps=1e-6, wide=True, interleaved=True)
