"""Pins of the serving-step oracle by properties that the mathematics fixes (CPU)."""
import numpy as np

import oracle
from oracle import serving


def _bits(x):
    return (np.asarray(x, dtype=np.float32).view(np.uint32) >> 16).astype(np.uint16)


def test_assign_by_hand():
    table = np.full((3, 2, 3), -1)
    table[0, :, 0] = [5, 6]
    a = serving.assign_slots([2, 0, 65], 70, [63, 10, 0], table, [1, 2, 3, 4, 7, 8, 9], 10)
    # request 0: position 63 in its block, position 64 opens a block with pages 9, 8
    assert a["slot_map"][:2].tolist() == [[5 * 64 + 63, 6 * 64 + 63], [9 * 64, 8 * 64]]
    # request 2: two blocks, pages 7, 4 then 3, 2
    assert a["page_table"][2].tolist() == [[7, 3, -1], [4, 2, -1]]
    assert a["positions"][2:67].tolist() == list(range(65)) and a["free"] == [1]
    assert a["token_indptr"].tolist() == [0, 2, 2, 67]
    assert a["slot_map"][67:].tolist() == [[-1, -1]] * 3


def test_assign_refusals():
    table = np.full((4, 1, 2), 0)
    a = serving.assign_slots([-1, 129, 64, 3], 200, [0, 0, 64, 5], table, [], 1)
    assert a["granted"].tolist() == [0, 0, 0, 3]     # no pages left, but 3 more fit in a held one
    assert a["seq_len"].tolist() == [0, 0, 64, 8]
    assert a["positions"][193:196].tolist() == [5, 6, 7]


def test_release_then_assign_keeps_every_page():
    rng = np.random.default_rng(0)
    B, H, most = 6, 2, 5
    lens = rng.integers(0, 300, B)
    order = list(rng.permutation(200))
    table = np.full((B, H, most + 2), -1)
    for b in range(B):
        for j in range(-(-lens[b] // 64)):
            for h in range(H):
                table[b, h, j] = order.pop()
    lens2, free = serving.release_pages([1, 0, 0, 1, 0, 0], lens, table, order, 200, most + 2)
    a = serving.assign_slots(rng.integers(0, 90, B), 600, lens2, table, free, 200)
    held = [a["page_table"][b, h, j] for b in range(B) for h in range(H)
            for j in range(-(-a["seq_len"][b] // 64))]
    assert sorted(held + a["free"]) == list(range(200))


def test_rotation_depends_on_distance():
    rng = np.random.default_rng(1)
    x, y = rng.normal(size=(2, 1, 1, 64))
    f = (10000.0 ** (-np.arange(32) / 32)).astype(np.float32)
    dots = []
    for base in (0, 7, 100000):
        a = serving.rotate(x, np.array([[base + 11]]), f)
        b = serving.rotate(y, np.array([[base]]), f)
        dots.append(float((a * b).sum()))
    assert np.ptp(dots) < 1e-9
    inter = serving.rotate(x, np.array([[3]]), f, interleaved=True)
    perm = np.arange(64).reshape(2, 32).T.ravel()       # (i, i + 32) pairs side by side
    assert np.allclose(inter[..., :], serving.rotate(x[..., np.argsort(perm)], np.array([[3]]), f)[..., perm])


def test_decode_equals_a_chunk_of_one_token():
    rng = np.random.default_rng(2)
    B, Hq, Hkv, D, lens = 2, 4, 2, 64, [130, 65]
    table = rng.permutation(B * Hkv * 3).reshape(B, Hkv, 3).astype(np.int32)
    q, k, v = (_bits(rng.normal(size=s)) for s in ((B, Hq, D), (12, 64, D), (12, 64, D)))
    out, lse, mass, _ = serving.decode_attention(q, k, v, table, lens, 0.125)
    T = [[[0, 1, 2]] * Hkv, [[0, 1]] * Hkv]
    ref, ref_lse = oracle.chunk_attention(q[:, None], k, v, table, np.array(lens) - 1, T, 2, 0.125)
    assert np.allclose(out, ref[:, 0]) and np.allclose(lse, ref_lse[..., 0])
    assert (mass >= np.abs(out) - 1e-12).all()
