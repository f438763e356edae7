"""A beam search as a server runs it: prompts, forks, decode steps over shared prefixes, reordered beams, a
compaction in between; eagerly, and with every call captured once and replayed.

A model on the host keeps every request's tokens as they were given.  After every step the cache must hold
them: values bit for bit, keys normalised and turned, within 2^-19 of each element of a pair for the norm, 2^-20
of both for the turn, and a bf16 half step.  The attention's tolerance is that of test_gpu_prefix.py, over
the keys and values that the cache holds, each request's by its own row of the page table.
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
NAMES = ("seq_len", "page_table", "page_shares", "free_pages", "free_count")


def _bf16(rng, shape, scale=1.0):
    return synth.bf16_round((rng.standard_normal(shape) * scale).astype(np.float32))


def _bits(t):
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


class Server:
    def __init__(self, rng, layout, D, graphs):
        self.rng, self.layout, self.D, self.graphs = rng, layout, D, graphs
        self.B, self.Hq, self.Hkv, self.most, self.pages, self.eps = 6, 8, 2, 12, 160, 1e-5
        B, Hkv, pages = self.B, self.Hkv, self.pages
        self.c = ca.Cache(B, self.Hq, Hkv, D, self.most, pages, v_layout=layout)
        order = rng.permutation(pages)
        self.d = dict(seq_len=i32_dev(np.zeros(B)), page_table=i32_dev(np.full((B, Hkv, self.most), -1)),
                      page_shares=i32_dev(np.zeros(pages)), free_pages=i32_dev(order), free_count=i32_dev([pages]))
        # pages start with NaN, which no one may read
        self.pools = tuple(bf16_dev(np.full(s, 0x7fc0, np.uint16)) for s in (self.c._k_pool, self.c._v_pool))
        self.f = (10000.0 ** (-np.arange(D // 2) / (D // 2))).astype(np.float32)
        self.w = [_bf16(rng, D, 0.3) for _ in "qk"]
        self.r = ca.Rotary(torch.from_numpy(self.f).to(DEV), norm=ca.HeadNorm(*map(bf16_dev, self.w), eps=self.eps))
        self.hist = [[] for _ in range(B)]
        self.parent, self.new = i32_dev(np.full(B, -1)), i32_dev(np.ones(B))
        self.share, self.share_len = i32_dev([0, 0, 0, 0, 1, 1]), i32_dev([0, 0])
        self.x = bf16_dev(np.zeros((B, self.Hq + 2 * Hkv, D), np.uint16))
        self.out, self.lse = torch.zeros(B, self.Hq, D, device=DEV, dtype=torch.bfloat16), torch.zeros(B, self.Hq, device=DEV)
        self.q = torch.zeros_like(self.out)
        self.slots = dict(seq_len=self.d["seq_len"], free_count=self.d["free_count"])
        # graphs that never run at once share a workspace
        n = max(ca.sharing.fork_workspace_bytes(self.c), ca.sharing.compact_workspace_bytes(self.c),
                ca.sharing.prefix_decode_workspace_bytes(self.c, 2))
        self.ws = torch.full((n,), 0xff, dtype=torch.uint8, device=DEV)
        self.captured = {}

    def call(self, name, fn):
        if not self.graphs:
            return fn()
        if name not in self.captured:
            keep = {k: t.clone() for k, t in self.d.items()}, [p.clone() for p in self.pools]
            fn()                       # outputs are made, libraries are loaded
            for k, t in self.d.items():
                t.copy_(keep[0][k])
            for p, was in zip(self.pools, keep[1]):
                p.copy_(was)
            torch.cuda.synchronize()
            self.captured[name] = torch.cuda.CUDAGraph()
            with torch.cuda.graph(self.captured[name]):
                fn()
        self.captured[name].replay()

    def prompt(self, lens):
        T, rows = sum(lens), self.Hq + 2 * self.Hkv
        x = _bf16(self.rng, (T + 3, rows, self.D), 2.0)       # three rows of padding belong to no one
        a = ca.assign_slots(self.c, i32_dev(lens), T + 3, *[self.d[k] for k in ("seq_len", "page_table", "free_pages", "free_count")],
                            dict(self.slots))
        t = bf16_dev(x)
        self._append(t, a, None)
        at = 0
        for b, n in enumerate(lens):
            self.hist[b] += [x[i] for i in range(at, at + n)]
            at += n

    def _append(self, t, a, out):
        Hq, Hkv = self.Hq, self.Hkv
        return ca.rotary_append(self.c, self.r, t[:, :Hq], t[:, Hq:Hq + Hkv], t[:, Hq + Hkv:], a["positions"], a["slot_map"],
                                self.pools, out=out)

    def fork(self, parent):
        self.parent.copy_(i32_dev(parent))
        self.call("fork", lambda: ca.sharing.fork_requests(self.c, self.parent, *[self.d[k] for k in NAMES], self.pools,
                                                           bufs=dict(self.d), ws=self.ws))
        self.hist = [[] if p < 0 else list(self.hist[p]) for p in parent]

    def compact(self):
        names = NAMES[1:]
        self.call("compact", lambda: ca.sharing.compact_pages(self.c, *[self.d[k] for k in NAMES], self.pools,
                                                              bufs=dict({k: self.d[k] for k in names}), ws=self.ws))

    def step(self):
        x = _bf16(self.rng, tuple(self.x.shape), 2.0)
        self.x.copy_(bf16_dev(x))

        def run():
            ca.assign_slots(self.c, self.new, self.B, *[self.d[k] for k in ("seq_len", "page_table", "free_pages", "free_count")],
                            self.slots)
            self._append(self.x, self.slots, self.q)
            ca.sharing.prefix_decode_attention(self.c, self.q, self.pools, self.d["page_table"], self.d["seq_len"], self.share,
                                               self.share_len, self.D ** -0.5, out=self.out, lse=self.lse, ws=self.ws)

        self.call("step", run)
        for b in range(self.B):
            self.hist[b].append(x[b])

    def check(self, attended):
        torch.cuda.synchronize()
        lens, table = self.d["seq_len"].cpu().numpy(), self.d["page_table"].cpu().numpy()
        assert lens.tolist() == [len(h) for h in self.hist]
        kp, vp = map(_bits, self.pools)
        if self.layout:
            vp = np.ascontiguousarray(vp.transpose(0, 2, 1))
        held = {}
        kw = oracle.bf16_to_f64(self.w[1])
        for b, h in enumerate(self.hist):
            n = len(h)
            for kvh in range(self.Hkv):
                ids = table[b, kvh, :-(-n // 64)]
                for p in ids:
                    held[int(p)] = held.get(int(p), 0) + 1
                if n == 0:
                    continue
                at = np.arange(n)
                x = np.stack(h)
                assert np.array_equal(vp[ids[at // 64], at % 64], x[:, self.Hq + self.Hkv + kvh])
                y = sharing.normed(oracle.bf16_to_f64(x[:, self.Hq + kvh]), kw, self.eps)
                want = serving.rotate(y[:, None], at[None], self.f)[:, 0]
                both = np.abs(y).reshape(n, 2, -1).sum(1)
                tol = BF16_HALF * np.abs(want) + np.tile(both, 2) * (2.0 ** -19 + 2.0 ** -20)
                assert (np.abs(oracle.bf16_to_f64(kp[ids[at // 64], at % 64]) - want) <= tol).all()
        # holds: every page once, those of several requests counted, the others free
        shares, free = self.d["page_shares"].cpu().numpy(), self.d["free_pages"].cpu().numpy()[:int(self.d["free_count"])]
        assert sorted(list(held) + free.tolist()) == list(range(self.pages))
        assert all(shares[p] == held.get(p, 1) - 1 for p in range(self.pages))
        if attended:
            ref, ref_lse, mass, size = serving.decode_attention(_bits(self.q), kp, vp, table, lens, self.D ** -0.5)
            delta = self.D * 2.0 ** -23 * size[..., None]
            err = np.abs(bf16_host_f64(self.out) - ref)
            assert (err <= BF16_HALF * np.abs(ref) + (2.0 ** -16 + 2 * delta + 2.0 ** -19) * mass).all()
            assert (np.abs(self.lse.cpu().numpy() - ref_lse) <= delta[..., 0] + 2.0 ** -19 * np.maximum(1, np.abs(ref_lse))).all()


@pytest.mark.parametrize("layout,D", [(0, 128), (1, 64)])
@pytest.mark.parametrize("graphs", [False, True])
def test_beam_search(layout, D, graphs):
    rng = np.random.default_rng(31 + layout)
    s = Server(rng, layout, D, graphs)
    prompts = [330, 0, 0, 0, 126, 0]
    s.prompt(prompts)
    s.check(False)
    s.share_len.copy_(i32_dev([330, 126]))
    s.fork([0, 0, 0, 0, 4, 4])
    s.check(False)
    moves = [[0, 1, 2, 3, 4, 5], [1, 1, 3, 0, 5, 5], [3, 2, 2, 2, 4, 5], [0, 0, 0, 0, 5, 4]]
    for i in range(8):
        s.step()
        s.check(True)
        s.fork(moves[i % 4])
        if i in (3, 6):
            s.compact()
            top = int(s.pages - s.d["free_count"])
            assert s.d["free_pages"].cpu().tolist()[:s.pages - top] == list(range(s.pages - 1, top - 1, -1))
        s.check(False)
    s.fork([-1] * 6)
    s.check(False)
    assert int(s.d["free_count"]) == s.pages
