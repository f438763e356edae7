"""Decode attention over a workspace that holds anything: the counts of earlier launches too whose
pieces never came together."""
import numpy as np
import pytest
import torch

import synth
from _helpers import bf16_dev, i32_dev

pytestmark = pytest.mark.gpu

ca = pytest.importorskip("paper_2605_16839_amd")
DEV = "cuda"


def _bf16(rng, shape):
    return bf16_dev(synth.bf16_round(rng.standard_normal(shape).astype(np.float32)))


def _args(lens, Hq, Hkv, D):
    rng = np.random.default_rng(Hq + D)
    most = max(-(-n // 64) for n in lens)
    pages = 4 * most
    c = ca.Cache(len(lens), Hq, Hkv, D, most, pages)
    return (c, _bf16(rng, (len(lens), Hq, D)), (_bf16(rng, (pages, 64, D)), _bf16(rng, (pages, 64, D))),
            i32_dev(rng.integers(0, pages, (len(lens), Hkv, most))), i32_dev(lens), D ** -0.5)


# more than 8 rows, several workgroups to each: the last of them joins the row
CASES = [([20001] + [0] * 8, 4, 1, 64), ([9000, 30000, 64, 5], 8, 4, 128)]


@pytest.mark.parametrize("lens,Hq,Hkv,D", CASES)
def test_counts_of_another_launch(lens, Hq, Hkv, D):
    args = _args(lens, Hq, Hkv, D)
    want, _ = ca.decode_attention(*args)
    n = ca.decode_workspace_bytes(args[0])
    assert n % 8 == 0
    ws = torch.empty(n // 8, dtype=torch.int64, device=DEV)
    for pieces in (1, 2, 3, 5, 255):
        for one in ([0x5ca1ab1e0dd50000 + pieces] * 256,
                    # every counter another launch's: 0, 1, ..
                    [pieces * (0xa7 << 56 | i << 16 | 1) % 2 ** 64 for i in range(256)]):
            ws.copy_(torch.from_numpy(np.resize(np.array(one, dtype=np.uint64), n // 8).view(np.int64)))
            for _ in range(2):
                out = torch.full_like(want, 7.0)
                ca.decode_attention(*args, out=out, ws=ws)
                assert torch.equal(out, want), (pieces, hex(one[0]))


@pytest.mark.parametrize("lens,Hq,Hkv,D", CASES)
def test_any_bytes(lens, Hq, Hkv, D):
    args = _args(lens, Hq, Hkv, D)
    want, _ = ca.decode_attention(*args)
    ws = torch.empty(ca.decode_workspace_bytes(args[0]), dtype=torch.uint8, device=DEV)
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    for fill in (0, 1, 0x7f, 0x80, 0xfe, 0xff, None, None, None):
        if fill is None:
            ws.copy_(torch.randint(0, 256, ws.shape, generator=g, device=DEV, dtype=torch.uint8))
        else:
            ws.fill_(fill)
        for _ in range(2):
            assert torch.equal(ca.decode_attention(*args, ws=ws)[0], want), fill
    # values below 0: the adds of pieces bring such a counter through 0
    few = torch.arange(ws.numel() // 8, device=DEV, dtype=torch.int64) % 9
    ws.view(torch.int64).copy_(-few * (0xa7 << 40 | 1) * 65536 - few)
    assert torch.equal(ca.decode_attention(*args, ws=ws)[0], want)


def test_a_workspace_of_zeros_before_a_replay():
    args = _args(*CASES[0])
    want, _ = ca.decode_attention(*args)
    ws = torch.zeros(ca.decode_workspace_bytes(args[0]), dtype=torch.uint8, device=DEV)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out, _ = ca.decode_attention(*args, ws=ws)
    for i in range(4):
        if i == 2:
            ws.zero_()
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        assert torch.equal(ca.decode_attention(*args, ws=ws)[0], want)
