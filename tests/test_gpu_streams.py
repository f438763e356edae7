"""Calls on streams given by argument that make their own workspaces and outputs, while the
caller's stream goes on using memory."""
import numpy as np
import pytest
import torch

from _helpers import bf16_dev, i32_dev
import synth

pytestmark = pytest.mark.gpu

ca = pytest.importorskip("paper_2605_16839_amd")
DEV = "cuda"


def _bf16(rng, shape):
    return bf16_dev(synth.bf16_round(rng.standard_normal(shape).astype(np.float32)))


def _case(rng, lens, Hq, Hkv, D):
    most = max(-(-n // 64) for n in lens)
    pages = len(lens) * Hkv * most
    c = ca.Cache(len(lens), Hq, Hkv, D, most, pages)
    table = i32_dev(rng.permutation(pages).reshape(len(lens), Hkv, most))
    return c, (_bf16(rng, (pages, 64, D)), _bf16(rng, (pages, 64, D))), table, i32_dev(lens)


def test_decode_on_two_streams_with_workspaces_of_its_own():
    rng = np.random.default_rng(1)
    c, pools, table, lens = _case(rng, [20000, 9000, 64], 8, 2, 64)
    q = [_bf16(rng, (3, 8, 64)) for _ in range(2)]
    want = [ca.decode_attention(c, x, pools, table, lens, 0.125)[0] for x in q]
    n = ca.decode_workspace_bytes(c)
    streams = [torch.cuda.Stream() for _ in q]
    torch.cuda.synchronize()
    got = []
    for i in range(6):
        for x, st in zip(q, streams):
            with torch.cuda.stream(st):
                torch.cuda._sleep(2_000_000)
            got.append(ca.decode_attention(c, x, pools, table, lens, 0.125, stream=st)[0])
            # memory that the caller's stream takes meanwhile, of the workspace's size and the output's
            for size in (n, x.numel() * 2):
                torch.empty(size, dtype=torch.uint8, device=DEV).fill_(0x41 + i)
    torch.cuda.synchronize()
    for i, x in enumerate(got):
        assert torch.equal(x, want[i % 2]), i


def test_append_and_slots_on_a_stream_with_outputs_of_their_own():
    rng = np.random.default_rng(2)
    Hq, Hkv, D, T = 4, 2, 64, 130
    c, pools, _, _ = _case(rng, [200, 200], Hq, Hkv, D)
    table, free = torch.full((2, Hkv, 4), -1, dtype=torch.int32, device=DEV), i32_dev(np.arange(c.num_pages))
    new, zero, count = i32_dev([100, 30]), i32_dev([0, 0]), i32_dev([c.num_pages])
    qkv = _bf16(rng, (T, Hq + 2 * Hkv, D))
    rot = ca.Rotary((1e4 ** (-torch.arange(D // 2, device=DEV) / (D // 2))).float())
    parts = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]

    def step(**kw):
        b = ca.assign_slots(c, new, T, zero, table, free, count, **kw)
        return b, ca.rotary_append(c, rot, *parts, b["positions"], b["slot_map"], pools, **kw)

    want, wq = step()
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = []
    for i in range(5):
        with torch.cuda.stream(st):
            torch.cuda._sleep(2_000_000)
        got.append(step(stream=st))
        for size in (8 * T * Hkv, 4 * (T + 8), wq.numel() * 2):
            torch.empty(size, dtype=torch.uint8, device=DEV).fill_(0x41)
    torch.cuda.synchronize()
    for b, q in got:
        assert torch.equal(q, wq) and all(torch.equal(b[k], want[k]) for k in want)
