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
