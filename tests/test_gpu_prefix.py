"""Decode attention over shared prefixes against the float64 oracle.

Tolerance as in test_gpu_serving.py: a score sums D exact products in fp32, off by at most delta = D * 2^-23
* max_j sm_scale sum_d |q_d k_jd|; a weight by 2 delta, by 2^-20 for exponential and rescaling, and by the
2^-16 of its two bf16 parts; the join of a row's pieces adds sums of weights in fp32, 2^-20 of them more.  All
of it scales sum_j w_j |v_j|; the store rounds to bf16, 2^-8 at most.
"""
import numpy as np
import pytest
import torch

import synth
from _helpers import bf16_dev, bf16_host_f64, i32_dev
from oracle import serving, sharing

pytestmark = pytest.mark.gpu

ca = pytest.importorskip("paper_2605_16839_amd")
DEV = "cuda"
BF16_HALF = 2.0 ** -8


def _bf16(rng, shape, scale=1.0):
    return synth.bf16_round((rng.standard_normal(shape) * scale).astype(np.float32))


def _cache(rng, share, share_len, lens, Hkv, D, max_blocks, poison=True, same=True):
    """Pools and a table whose members' rows name the first member's pages (same), or pages of their own
    (which no one may read); NaN and infinities behind every request's last token."""
    B = len(lens)
    blocks = [-(-max(n, 0) // 64) for n in lens]
    pages = sum(blocks) * Hkv + 2
    order = list(rng.permutation(pages))
    table = rng.choice([-1, pages, 2**31 - 1, 0], (B, Hkv, max_blocks))
    kp, vp = _bf16(rng, (pages, 64, D)), _bf16(rng, (pages, 64, D))
    for b, n in enumerate(lens):
        for j in range(blocks[b]):
            for h in range(Hkv):
                p = table[b, h, j] = order.pop()
                if poison and n - 64 * j < 64:
                    kp[p, n - 64 * j:] = rng.choice([0x7fc0, 0x7f80, 0xff80])
                    vp[p, n - 64 * j:] = rng.choice([0x7fc0, 0x7f80, 0xff80])
    rows = sharing.prefix_rows(table, lens, share, share_len)
    return kp, vp, rows if same else table, rows, pages


def _ok(out, lse, q, kp, vp, rows, lens, scale):
    ref, ref_lse, mass, size = serving.decode_attention(q, kp, vp, rows, lens, scale)
    D = q.shape[-1]
    delta = D * 2.0 ** -23 * size[..., None]
    got = bf16_host_f64(out)
    assert np.isfinite(got).all()
    err = np.abs(got - ref)
    tol = BF16_HALF * np.abs(ref) + (2.0 ** -16 + 2 * delta + 2.0 ** -19) * mass
    assert (err <= tol).all(), (np.max(err - tol), np.argwhere(err > tol)[:5])
    gl = lse.cpu().numpy().astype(np.float64)
    fin = np.isfinite(ref_lse)
    assert np.array_equal(np.isfinite(gl), fin) and (gl[~fin] == -np.inf).all()
    assert (np.abs(gl[fin] - ref_lse[fin]) <= delta[..., 0][fin] + 2.0 ** -19 * np.maximum(1, np.abs(ref_lse[fin]))).all()


def _run(rng, share, share_len, lens, Hq, Hkv, D, layout=0, max_blocks=None, same=True, qscale=2.0, scale=None):
    max_blocks = max_blocks or max(1, max(-(-n // 64) for n in lens))
    kp, vp, table, rows, pages = _cache(rng, share, share_len, lens, Hkv, D, max_blocks, same=same)
    q = _bf16(rng, (len(lens), Hq, D), qscale)
    scale = scale or D ** -0.5
    c = ca.Cache(len(lens), Hq, Hkv, D, max_blocks, pages, v_layout=layout)
    vd = vp if layout == 0 else synth.v_pages_transposed(vp)
    lse = torch.full((len(lens), Hq), 7.0, device=DEV)
    out = torch.full((len(lens), Hq, D), 9.0, device=DEV, dtype=torch.bfloat16)
    n = ca.sharing.prefix_decode_workspace_bytes(c, len(share_len))
    ws = torch.full((n,), 0xff, dtype=torch.uint8, device=DEV)
    args = (c, bf16_dev(q), (bf16_dev(kp), bf16_dev(vd)), i32_dev(table), i32_dev(lens), i32_dev(share),
            i32_dev(share_len), scale)
    ca.sharing.prefix_decode_attention(*args, out=out, lse=lse, ws=ws)
    torch.cuda.synchronize()
    _ok(out, lse, q, kp, vp, rows, lens, scale)
    again, _ = ca.sharing.prefix_decode_attention(*args)      # the same bits again, another workspace, no lse
    assert torch.equal(again, out)


def _behind(share, share_len, mine):
    return [m if s < 0 else share_len[s] + m for s, m in zip(share, mine)]


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("Hq,Hkv,D", [(4, 1, 64), (32, 8, 128), (8, 8, 64), (28, 4, 128), (9, 1, 128), (16, 1, 64),
                                      (40, 1, 64), (71, 1, 128), (300, 1, 64), (513, 1, 128), (1, 1, 128)])
def test_heads(Hq, Hkv, D, layout):
    rng = np.random.default_rng(Hq * 7 + D)
    share, share_len = [0, 1, -1, 0, 0, 1, 0, 2], [200, 700, 64]
    _run(rng, share, share_len, _behind(share, share_len, [1, 64, 300, 0, 63, 65, 129, 10]), Hq, Hkv, D, layout)


@pytest.mark.parametrize("B", [1, 2, 7, 8, 15, 16, 17, 31, 33, 40, 63, 64, 65, 70, 129])
def test_members(B):
    """Rows of a share on both sides of what a wave and a tile hold (4 heads on a KV head)."""
    rng = np.random.default_rng(B)
    for D, layout in ((64, 1), (128, 0)):
        _run(rng, [0] * B, [330], [330 + int(n) for n in rng.integers(0, 100, B)], 4, 1, D, layout)


@pytest.mark.parametrize("share,share_len,mine,Hkv,max_blocks", [
    ([0], [64], [0], 1, None), ([0, 0], [64], [0, 0], 1, 1), ([0, 0], [63], [1, 64], 2, None),
    ([0, 0, 0], [128], [0, 0, 0], 8, 9), ([0, 0], [0], [5, 0], 1, None), ([-1, -1], [640], [3, 200], 2, None),
    ([0, 0, 0, 0], [20001], [1, 2, 70, 3000], 1, None), ([0, 1, 0, 1], [9000, 100], [1, 1, 1, 1], 2, 2048),
    ([1, 1, 1, 0, 0, 0], [64, 6400], [1, 64, 128, 200, 1, 9], 8, 400), ([2, 7, -5, 2**31 - 1], [64, 64, 64], [99, 1, 1, 1], 1, None),
    ([0] * 40, [65], [1] * 40, 8, None), ([i // 3 for i in range(90)], [64 * (i % 5) + 7 for i in range(30)], [i for i in range(90)], 2, None),
    ([0] * 3 + [1], [300, 300], [-300, 10, -300, -300], 2, 7),      # idle rows, named in a share
])
def test_lengths(share, share_len, mine, Hkv, max_blocks):
    rng = np.random.default_rng(len(share) + Hkv)
    lens = [m if not 0 <= s < len(share_len) else share_len[s] + m for s, m in zip(share, mine)]
    for layout in (0, 1):
        _run(rng, share, share_len, lens, 2 * Hkv, Hkv, 64 if len(lens) > 30 else 128, layout, max_blocks)


def test_shorter_than_the_share():
    """A request that does not hold all of the share's pages is taken by itself."""
    rng = np.random.default_rng(5)
    for lens in ([700, 639, 640, 1, 0, 641], [1, 700, 640, 640, 0, 0], [639, 640, 1, 0, 0, 0]):
        _run(rng, [0] * 6, [645], lens, 8, 2, 128, 0, same=True)


def test_the_first_members_pages_count():
    rng = np.random.default_rng(6)
    _run(rng, [0, 0, 1, 0, 1], [200, 640], [260, 200, 700, 300, 641], 8, 2, 128, 0, same=False)
    _run(rng, [0, 0, 1, 0, 1], [200, 640], [191, 200, 700, 300, 641], 8, 2, 64, 1, same=False)    # 0 is no member


def test_share_len_out_of_range():
    rng = np.random.default_rng(7)
    _run(rng, [0, 0, 1, 1], [-70, 2**31 - 1], [100, 130, 64, 60], 4, 2, 64, 0)
    _run(rng, [0, 0, 1, 1], [2**31 - 1, -2**31], [192, 192, 64, 60], 4, 2, 64, 0, max_blocks=3)


def test_no_shares_is_decode_attention():
    rng = np.random.default_rng(8)
    lens = [1, 0, 63, 700, 64, 2048]
    kp, vp, table, _, pages = _cache(rng, [-1] * 6, [], lens, 2, 128, 40)
    c = ca.Cache(6, 8, 2, 128, 40, pages)
    q, pools, pt, n = bf16_dev(_bf16(rng, (6, 8, 128))), (bf16_dev(kp), bf16_dev(vp)), i32_dev(table), i32_dev(lens)
    a, _ = ca.sharing.prefix_decode_attention(c, q, pools, pt, n, i32_dev([-1] * 6), i32_dev([]), 0.1)
    b, _ = ca.decode_attention(c, q, pools, pt, n, 0.1)
    # both are within a bf16 half step and a little of the exact result
    assert ((a.float() - b.float()).abs() <= 2.1 * BF16_HALF * b.float().abs() + 2.0 ** -14).all()


@pytest.mark.parametrize("B", [256, 1000, 2048])
def test_many_requests(B):
    rng = np.random.default_rng(B)
    share = rng.integers(-1, 512 if B > 1000 else 30, B).tolist()
    share_len = rng.integers(0, 200, 512 if B > 1000 else 30).tolist()
    idle = rng.random(B) < 0.5
    lens = [0 if i else (0 if s < 0 else share_len[s]) + int(m) for s, m, i in zip(share, rng.integers(1, 70, B), idle)]
    _run(rng, share, share_len, lens, 2, 1, 64, 0)


def test_missing_pages_and_bad_ids():
    """Ids out of range add no keys, in the prefix and behind it."""
    rng = np.random.default_rng(9)
    share, share_len, lens = [0, 0, 0], [256], [300, 320, 257]
    kp, vp, table, rows, pages = _cache(rng, share, share_len, lens, 2, 128, 5)
    for bad in (-1, pages, 2**31 - 1, -2**31):
        t = rows.copy()
        t[:, 0, 1], t[1, 1, 4] = bad, bad
        keep = kp, vp, np.where((t < 0) | (t >= pages), pages, t)      # a page of its own that no weight reaches
        q = _bf16(rng, (3, 8, 128), 2.0)
        c = ca.Cache(3, 8, 2, 128, 5, pages)
        lse = torch.empty(3, 8, device=DEV)
        out, _ = ca.sharing.prefix_decode_attention(c, bf16_dev(q), (bf16_dev(kp), bf16_dev(vp)), i32_dev(t), i32_dev(lens),
                                                    i32_dev(share), i32_dev(share_len), 0.1, lse=lse)
        # the oracle over lists of the blocks that are there
        lists = [[[j for j in range(-(-n // 64)) if 0 <= t[b, h, j] < pages] for h in range(2)] for b, n in enumerate(lens)]
        ref, ref_lse, mass, size = serving.decode_attention(q, kp, vp, np.minimum(keep[2], pages - 1), lens, 0.1, lists, 4)
        err = np.abs(bf16_host_f64(out) - ref)
        delta = 128 * 2.0 ** -23 * size[..., None]
        assert (err <= BF16_HALF * np.abs(ref) + (2.0 ** -16 + 2 * delta + 2.0 ** -19) * mass).all()
        assert np.allclose(lse.cpu().numpy(), ref_lse, rtol=2e-6, atol=2e-6)


@pytest.mark.parametrize("layout", [0, 1])
def test_not_finite(layout):
    """Scores of NaN or +inf give NaN and lse -inf, -inf adds nothing, infinities of v stay infinities."""
    rng = np.random.default_rng(10)
    share, share_len, lens = [0, 0, -1], [128], [200, 150, 70]
    kp, vp, table, rows, pages = _cache(rng, share, share_len, lens, 1, 64, 4, poison=False)
    kp &= 0x7fff                                   # keys >= 0, so a query >= 0 makes every score >= 0
    q = np.abs(rng.standard_normal((3, 2, 64))) + 0.1
    c = ca.Cache(3, 2, 1, 64, 4, pages, v_layout=layout)

    def call(k, v):
        lse = torch.empty(3, 2, device=DEV)
        vd = v if layout == 0 else synth.v_pages_transposed(v)
        out, _ = ca.sharing.prefix_decode_attention(c, bf16_dev(synth.bf16_round(q.astype(np.float32))), (bf16_dev(k), bf16_dev(vd)),
                                                    i32_dev(rows), i32_dev(lens), i32_dev(share), i32_dev(share_len), 0.125, lse=lse)
        return out.float().cpu().numpy(), lse.cpu().numpy()

    for block, hit in ((0, [0, 1]), (1, [0, 1]), (2, [0])):
        for bits in (0x7fc0, 0x7f80):
            k = kp.copy()
            k[rows[0, 0, block], 5, 3] = bits
            out, lse = call(k, vp)
            for b in range(3):
                assert (np.isnan(out[b]).all() and (lse[b] == -np.inf).all()) == (b in hit)
                assert np.isfinite(out[b]).all() == (b not in hit)
        k = kp.copy()
        k[rows[0, 0, block], 5, 3] = 0xff80          # a score of -inf
        out, lse = call(k, vp)
        assert np.isfinite(out).all() and np.isfinite(lse).all()
        for bits, value in ((0x7f80, np.inf), (0xff80, -np.inf), (0x7fc0, np.nan)):
            v = vp.copy()
            v[rows[0, 0, block], 9, 11] = bits
            out, lse = call(kp, v)
            assert np.isfinite(lse).all()
            for b in range(3):
                want = np.zeros((2, 64), bool)
                want[:, 11] = b in hit
                assert np.array_equal(~np.isfinite(out[b]), want)
                if b in hit:
                    assert np.array_equal(out[b][:, 11], [value, value], equal_nan=True)


def test_far_scores():
    """Large scores of growing size, so that the maximum moves in every page and piece."""
    rng = np.random.default_rng(11)
    share, share_len = [0, 0, 0], [4000]
    for qs in (0.0, 30.0):
        _run(rng, share, share_len, [4100, 4001, 4500], 4, 1, 128, 0, qscale=qs)


def test_in_a_graph_on_a_stream_two_at_once():
    """Replayed with other lengths and shares; two calls at once on two workspaces."""
    rng = np.random.default_rng(12)
    B, Hq, Hkv, D, most = 9, 8, 2, 64, 12
    share_len = [300, 128]
    sets = []
    for i in range(3):
        share = rng.integers(-1, 2, B).tolist()
        mine = rng.integers(0, 200, B)
        lens = [int(m) + (share_len[s] if s >= 0 else 0) for s, m in zip(share, mine)]
        sets.append((share, lens))
    pages = 300
    kp, vp = _bf16(rng, (pages, 64, D)), _bf16(rng, (pages, 64, D))
    table = rng.integers(0, pages, (B, Hkv, most))
    c = ca.Cache(B, Hq, Hkv, D, most, pages)
    q = bf16_dev(_bf16(rng, (B, Hq, D)))
    pools, pt = (bf16_dev(kp), bf16_dev(vp)), i32_dev(table)
    sh, ln, sl = i32_dev(sets[0][0]), i32_dev(sets[0][1]), i32_dev(share_len)
    lse, out = torch.empty(B, Hq, device=DEV), torch.empty_like(q)
    n = ca.sharing.prefix_decode_workspace_bytes(c, 2)
    ws, ws2 = (torch.zeros(n, dtype=torch.uint8, device=DEV) for _ in "ab")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other, _ = ca.sharing.prefix_decode_attention(c, q, pools, pt, ln, sh, sl, 0.2, ws=ws2, stream=side)
    one, _ = ca.sharing.prefix_decode_attention(c, q, pools, pt, ln, sh, sl, 0.2, ws=ws)
    torch.cuda.synchronize()
    assert torch.equal(one, other)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ca.sharing.prefix_decode_attention(c, q, pools, pt, ln, sh, sl, 0.2, out=out, lse=lse, ws=ws)
    for share, lens in sets * 2:
        sh.copy_(i32_dev(share))
        ln.copy_(i32_dev(lens))
        g.replay()
        torch.cuda.synchronize()
        rows = sharing.prefix_rows(table, lens, share, share_len)
        _ok(out, lse, np.ascontiguousarray(q.view(torch.int16).cpu().numpy().view(np.uint16)), kp, vp, rows, lens, 0.2)


def test_binding_refuses():
    c = ca.Cache(2, 4, 2, 64, 3, 9)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)  # noqa: E731
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device=DEV)  # noqa: E731
    pools = (bf(9, 64, 64), bf(9, 64, 64))
    good = dict(q=bf(2, 4, 64), kv_pool=pools, page_table=i32(2, 2, 3), kv_len=i32(2), share=i32(2), share_len=i32(1))
    ca.sharing.prefix_decode_attention(c, **good, sm_scale=0.1)
    for k, v in (("q", bf(2, 4, 128)), ("page_table", i32(2, 2, 4)), ("kv_len", i32(3)), ("share", i32(3)),
                 ("share", i32(2).long()), ("share_len", i32(1).float()), ("kv_pool", (pools[0], bf(8, 64, 64)))):
        with pytest.raises(ValueError):
            ca.sharing.prefix_decode_attention(c, **{**good, k: v}, sm_scale=0.1)
    state = (i32(2), i32(2, 2, 3), i32(9), i32(9), i32(1))
    for i in range(5):
        bad = list(state)
        bad[i] = i32(4, 5)
        with pytest.raises(ValueError):
            ca.sharing.fork_requests(c, i32(2), *bad, pools)
    with pytest.raises(ValueError):
        ca.sharing.fork_requests(c, i32(2), *state, pools, keep_len=i32(3))
    with pytest.raises(ca.CAError, match="free_capacity"):
        ca.sharing.fork_requests(c, i32(2), *state[:3], i32(8), i32(1), pools)
    with pytest.raises(ValueError, match="come together"):
        ca.sharing.compact_pages(c, state[0], state[1], None, state[3], state[4], pools, bufs=dict(page_shares=i32(9)))


@pytest.mark.parametrize("layout", [0, 1])
def test_shares_of_all_sizes_in_one_call(layout):
    """Few and many rows to a page one after another, tiles of more than 256 rows, pairs' own pages behind them;
    from enough pages on that they are dealt by their cost, and more than a workgroup looks up together."""
    rng = np.random.default_rng(13)
    share = [0] * 3 + [1] * 40 + [2] * 2 + [3] * 20 + [-1] * 2 + [4] * 66
    share_len = [700, 900, 64 * 30, 1300, 130]
    order = rng.permutation(len(share))
    share = [share[i] for i in order]
    mine = rng.integers(0, 260, len(share)).tolist()
    mine[3], mine[20] = 5000, 1
    _run(rng, share, share_len, _behind(share, share_len, mine), 8, 2, 64, layout)
    _run(rng, share, share_len, _behind(share, share_len, mine), 14, 1, 128, layout)
    few = [0, 1, 0, -1, 1, 1, 0]
    _run(rng, few, [64 * 700, 64 * 650], _behind(few, [64 * 700, 64 * 650], [1, 5000, 70, 30000, 64, 1, 0]), 40, 1, 64, layout)


@pytest.mark.parametrize("far", [3, 20, 103, 104, 110, 112, 118, 125])
def test_infinities_behind_small_weights(far):
    """A weight of 2^-far, with no bits in its second part, still hands an infinity on, and only to its dimension."""
    rng = np.random.default_rng(far)
    share, share_len, lens = [0, 0, 0], [128], [200, 150, 131]
    for layout, D, Hq in ((0, 64, 2), (1, 128, 100)):
        kp, vp, table, rows, pages = _cache(rng, share, share_len, lens, 1, D, 4, poison=False)
        kp[:] = 0
        q = np.zeros((3, Hq, D), np.float32)
        q[:, :, 0] = 1
        for block, hit in ((1, [0, 1, 2]), (2, [1])):
            b = hit[0] if block == 1 else 1
            k, v = kp.copy(), vp.copy()
            k[rows[b, 0, block], 2, 0] = synth.bf16_round(np.float32([-far]))[0]
            v[rows[b, 0, block], 2, 7] = 0x7f80
            c = ca.Cache(3, Hq, 1, D, 4, pages, v_layout=layout)
            out, _ = ca.sharing.prefix_decode_attention(
                c, bf16_dev(synth.bf16_round(q)), (bf16_dev(k), bf16_dev(v if layout == 0 else synth.v_pages_transposed(v))),
                i32_dev(rows), i32_dev(lens), i32_dev(share), i32_dev(share_len), float(np.log(2.0)))
            out = out.float().cpu().numpy()
            want = np.zeros((3, Hq, D), bool)
            want[hit, :, 7] = True
            assert np.array_equal(np.isposinf(out), want) and np.isfinite(out[~want]).all()


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("D,Hq,members", [(64, 2, 3), (128, 4, 2), (128, 40, 2), (64, 100, 3), (128, 12, 20)])
def test_keys_without_weight_add_nothing(D, Hq, members, layout):
    """Scores of -inf, and scores so far below the largest that the weight is 0, meet values near the largest bf16:
    half of the prefix's keys and of each request's own."""
    rng = np.random.default_rng(D + Hq)
    share, share_len = [0] * members, [128]
    lens = [128 + int(n) for n in rng.integers(60, 100, members)]
    kp, vp, table, rows, pages = _cache(rng, share, share_len, lens, 1, D, 4, poison=False)
    q = np.zeros((members, Hq, D), np.float32)
    q[:, :, 0] = 1
    far = rng.random((pages, 64)) < 0.5
    vp[far] = synth.bf16_round(rng.choice(np.float32([3.3e38, -3.3e38]), (int(far.sum()), D)))
    for b in range(members):
        far[rows[b, 0, [0, 2]], 3] = False          # every request keeps a key of either kind
    for score in (0xff80, synth.bf16_round(np.float32([-300]))[0], synth.bf16_round(np.float32([-3e38]))[0]):
        k = np.zeros_like(kp)
        k[far, 0] = score
        v = vp.copy()
        v[~far & (np.abs(synth.bf16_bits_to_f32(vp[:, :, 0])) > 1e30)] = 0
        c = ca.Cache(members, Hq, 1, D, 4, pages, v_layout=layout)
        lse = torch.full((members, Hq), 7.0, device=DEV)
        out, _ = ca.sharing.prefix_decode_attention(
            c, bf16_dev(synth.bf16_round(q)), (bf16_dev(k), bf16_dev(v if layout == 0 else synth.v_pages_transposed(v))),
            i32_dev(rows), i32_dev(lens), i32_dev(share), i32_dev(share_len), float(np.log(2.0)), lse=lse)
        torch.cuda.synchronize()
        # the definition over the keys that have a weight: all have the score 0, so the mean of their values
        # (2^-300 of a value is below 2^-172).  Weights are 1 exactly, or 2^-8 at least where the maximum lags; their
        # sums take 2^-19 of the mass, as above.
        for b in range(members):
            n = lens[b]
            ids = rows[b, 0, np.arange(n) // 64]
            there = ~far[ids, np.arange(n) % 64]
            vals = synth.bf16_bits_to_f32(v[ids, np.arange(n) % 64]).astype(np.float64)[there]
            want, mass = vals.mean(0), np.abs(vals).mean(0)
            err = np.abs(bf16_host_f64(out[b]) - want)
            assert (err <= BF16_HALF * np.abs(want) + (2.0 ** -16 + 2.0 ** -19) * mass).all(), (score, b, err.max())
            assert np.abs(lse[b].cpu().numpy() - np.log(there.sum())).max() <= 2.0 ** -19 * np.log(there.sum())


def test_as_many_rows_as_a_launch_has_workgroups():
    """2^24 query rows and more: the join's workgroups of 256 threads are more than one launch takes.  A request
    with one key gets its value exactly, and lse 0 from a query of zeros."""
    g = torch.Generator(device=DEV)
    g.manual_seed(14)
    pages, D = 500, 64
    for B, Hq, Hkv in ((2048, 8192, 64), (2047, 257 * 32, 32)):
        c = ca.Cache(B, Hq, Hkv, D, 1, pages)
        kp, vp = (torch.randn((pages, 64, D), generator=g, device=DEV, dtype=torch.bfloat16) for _ in "kv")
        pt = torch.randint(0, pages, (B, Hkv, 1), generator=g, device=DEV, dtype=torch.int32)
        lens = (torch.arange(B, device=DEV) % 3 > 0).to(torch.int32)
        q = torch.zeros(B, Hq, D, device=DEV, dtype=torch.bfloat16)
        out, lse = torch.full_like(q, 9.0), torch.full((B, Hq), 7.0, device=DEV)
        none = torch.empty(0, dtype=torch.int32, device=DEV)
        ca.sharing.prefix_decode_attention(c, q, (kp, vp), pt, lens, torch.full_like(lens, -1), none, 0.1, out=out, lse=lse)
        torch.cuda.synchronize()
        for b in range(0, B, 256):
            some = slice(b, b + 256)
            want = vp[pt[some, :, 0].long(), 0] * lens[some, None, None].to(torch.bfloat16)
            got = out[some].view(-1, Hkv, Hq // Hkv, D)
            assert (got == want[:, :, None]).all()
            assert (lse[some] == torch.where(lens[some] > 0, 0.0, -float("inf"))[:, None]).all()
        del q, out, lse
