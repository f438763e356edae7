"""Decode attention: what the softmax weights lose does not depend on the number of heads.

A weight is held as two bf16, the second of what the first loses: off by 2^-8 of 2^-8.  A
score sums D exact products in fp32, off by at most delta = D * 2^-23 * max sm_scale sum_d |q_d k_jd|;
a weight by 2 delta and 2^-20 for the exponential.  All of it scales sum_j w_j |v_j|, and the
stored bf16 is off by 2^-8 of its value.
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


def _bf16(rng, shape, scale=1.0):
    return synth.bf16_round((rng.standard_normal(shape) * scale).astype(np.float32))


def _cache(rng, lens, Hkv, D):
    blocks = [-(-n // 64) for n in lens]
    most, pages = max(blocks), sum(blocks) * Hkv
    table, order = np.zeros((len(lens), Hkv, most), dtype=np.int64), iter(rng.permutation(pages))
    for b, n in enumerate(blocks):
        for j in range(n):
            for h in range(Hkv):
                table[b, h, j] = next(order)
    return _bf16(rng, (pages, 64, D)), _bf16(rng, (pages, 64, D)), table, pages


def _decode(q, kp, vp, table, lens, pages, scale, layout, tables=None, gs=0):
    B, Hq, D = q.shape
    c = ca.Cache(B, Hq, table.shape[1], D, table.shape[2], pages, v_layout=layout)
    vd = vp if layout == 0 else synth.v_pages_transposed(vp)
    lse = torch.empty(B, Hq, device=DEV)
    out, _ = ca.decode_attention(c, bf16_dev(q), (bf16_dev(kp), bf16_dev(vd)), i32_dev(table), i32_dev(lens),
                                 scale, tables=tables, group_size=gs, lse=lse)
    return bf16_host_f64(out), lse.cpu().numpy().astype(np.float64)


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("Hq,Hkv,D,gs", [(4, 1, 64, 0), (8, 1, 128, 0), (9, 1, 64, 0), (9, 1, 128, 0), (12, 1, 128, 0),
                                         (32, 2, 64, 0), (32, 2, 128, 0), (20, 1, 128, 0), (40, 1, 64, 0),
                                         (40, 1, 128, 20), (32, 2, 128, 8)])
def test_weights_keep_16_bits(Hq, Hkv, D, gs, layout):
    rng = np.random.default_rng(Hq + D)
    lens = [2, 3, 5, 64, 65, 1, 300, 2000]
    kp, vp, table, pages = _cache(rng, lens, Hkv, D)
    q = _bf16(rng, (len(lens), Hq, D))
    tables = lists = None
    if gs:
        lists = [[list(range(-(-n // 64))) for _ in range(Hq // gs)] for n in lens]
        rows = [r for t in lists for r in t]
        ix = np.zeros(len(rows) * table.shape[2])
        ip = np.concatenate([[0], np.cumsum([len(r) for r in rows])])
        ix[:ip[-1]] = [j for r in rows for j in r]
        tables = (i32_dev(ip), i32_dev(ix))
    scale = D ** -0.5
    got, lse = _decode(q, kp, vp, table, lens, pages, scale, layout, tables, gs)
    ref, ref_lse, mass, size = serving.decode_attention(q, kp, vp, table, lens, scale, lists, gs)
    delta = D * 2.0 ** -23 * size
    err = np.abs(got - ref)
    tol = BF16_HALF * np.abs(ref) + (2.0 ** -16 + 2 * delta[..., None] + 2.0 ** -20) * mass
    assert (err <= tol).all(), (float((err - tol).max()), np.argwhere(err > tol)[:4].tolist())
    assert (np.abs(lse - ref_lse) <= delta + 2.0 ** -20 * np.maximum(1, np.abs(ref_lse))).all()


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("Hq,Hkv,D", [(4, 1, 64), (8, 1, 128), (6, 2, 128), (9, 1, 128), (16, 1, 64), (20, 1, 64)])
def test_infinite_values(Hq, Hkv, D, layout):
    """out has the infinity of the values that it sums, NaN for both signs or a NaN, in rows of a
    page, of a wave's pages and of several workgroups' pieces."""
    rng = np.random.default_rng(Hq)
    lens = [1, 60, 300, 9000, 64 * 200]
    kp, vp, table, pages = _cache(rng, lens, Hkv, D)
    q = _bf16(rng, (len(lens), Hq, D), 0.5)      # every weight is far from 0
    inf, minus, nan = 0x7f80, 0xff80, 0x7fc0
    for b, n in enumerate(lens):
        for h in range(Hkv):
            def put(pos, d, bits):
                vp[table[b, h, pos // 64], pos % 64, d] = bits
            put(0, 1, inf), put(n - 1, 2, minus), put(n // 2, 3, nan)
            put(0, 5, inf), put(n - 1, 5, inf)
            put(n // 3, D - 1, minus)
            if n > 1:
                put(0, 7, inf), put(n - 1, 7, minus)
    scale = D ** -0.5
    got, lse = _decode(q, kp, vp, table, lens, pages, scale, layout)
    clean = np.where((vp & 0x7f80) == 0x7f80, np.uint16(0), vp)
    ref, ref_lse, mass, size = serving.decode_attention(q, kp, clean, table, lens, scale)
    with np.errstate(invalid="ignore"):
        raw = serving.decode_attention(q, kp, vp, table, lens, scale)[0]
    at = ~np.isfinite(raw)
    assert at[..., [1, 2, 3, 5, D - 1]].all() and np.isnan(raw[1:, :, 7]).all()
    assert np.array_equal(got[at], raw[at], equal_nan=True)
    delta = D * 2.0 ** -23 * size
    tol = BF16_HALF * np.abs(ref) + (2.0 ** -16 + 2 * delta[..., None] + 2.0 ** -20) * mass
    assert (np.abs(got - ref) <= tol)[~at].all()
    assert (np.abs(lse - ref_lse) <= delta + 2.0 ** -20 * np.maximum(1, np.abs(ref_lse))).all()
