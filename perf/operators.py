"""The work of a serving loop around the paged KV cache, as cases that can be timed and compared.

Between the prefill chunks of ``perf/cases.py`` a server decodes: every step it
gives the requests' new tokens their places in the cache (``release_pages`` of the
requests that ended, then ``assign_slots``), rotates the new queries and keys
and writes keys and values into the pages (``rotary_append``), and attends with
one query per request over the pages (``decode_attention``).  The same first two
calls carry a prefill chunk's tokens, before ``chunk_attention`` reads them.

Kinds of cases:
  decode  decode_attention, over the whole cache or over block tables
  append  rotary_append of the tokens of one step
  slots   release_pages (where requests ended) and assign_slots
"""
import math
import random

import torch

own = False   # set from outside: True runs this package's kernels, False the plain forms

PAGE = 64
DEVICE = "cuda"
ROPE_BASE = 500000.0   # of the LLaMA-3.1 layer that the workloads are shaped after


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------
def _decode(name, batch, shortest, longest, heads, dim, layout, density=1.0, group=0, idle=0, table_blocks=0,
            shape=1):
    """batch requests, idle of them empty (a graph captured for a larger batch than is
    running), the others of lengths spread over [shortest, longest] by their logarithm;
    density < 1: over block tables that list that part of the blocks."""
    c = dict(kind="decode", batch=batch, shortest=shortest, longest=longest, q_heads=heads[0],
             kv_heads=heads[1], dim=dim, layout=layout, density=density,
             group=group or heads[0] // heads[1], idle=idle, table_blocks=table_blocks, shape=shape)
    return dict(name=name, **c) if name else c


def _append(name, requests, tokens, longest, heads, dim, layout, rotary, axes=1, interleaved=False,
            padded=0, shape=1):
    """tokens new tokens of each request, whose cached lengths go up to longest; padded
    more rows belong to no request."""
    c = dict(kind="append", requests=requests, tokens=tokens, longest=longest, q_heads=heads[0],
             kv_heads=heads[1], dim=dim, layout=layout, rotary=rotary, axes=axes,
             interleaved=interleaved, padded=padded, shape=shape)
    return dict(name=name, **c) if name else c


def _slots(name, batch, longest, kv_heads, chunk, chunks, ended, padded=0, shape=1):
    """batch requests of cached lengths up to longest: chunks of them add chunk tokens
    (prefill), ended of them have ended, the others add one; padded rows more than the tokens."""
    c = dict(kind="slots", batch=batch, longest=longest, kv_heads=kv_heads, chunk=chunk,
             chunks=chunks, ended=ended, padded=padded, shape=shape)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # the smallest call: one request of a small model, where latency counts
        _decode("decode_small", 1, 700, 700, (4, 1), 64, "token_major"),
        # one user late in a 128K prompt: all CUs share one request's eight KV heads
        _decode("decode_one_long", 1, 131071, 131071, (32, 8), 128, "token_major",
                table_blocks=2048),
        # an ordinary batch of very different lengths, captured for 64 with 12 rows idle
        _decode("decode_batch", 64, 30, 16384, (32, 8), 128, "token_major", idle=12),
        # grouped queries of 8 heads per KV head, long contexts, transposed V pages
        _decode("decode_gqa8", 16, 20000, 60001, (32, 4), 128, "transposed"),
        # the largest call: a full batch of long contexts
        _decode("decode_large", 96, 4096, 32768, (32, 8), 128, "transposed", table_blocks=512),
        # long contexts over the selector's tables, a tenth of the blocks
        _decode("decode_selected", 8, 65536, 131000, (32, 8), 128, "token_major", density=0.1,
                table_blocks=2048),
        # one decode step's tokens, captured for 64 with 5 rows idle
        _append("append_decode", 59, 1, 32768, (32, 8), 128, "token_major", 128, padded=5),
        # four prefill chunks of 2048 tokens
        _append("append_chunks", 4, 2048, 126976, (32, 8), 128, "token_major", 128),
        # a prompt's remainder with image tokens: positions of three axes, transposed V pages
        _append("append_axes", 3, 1451, 50001, (32, 8), 128, "transposed", 128, axes=3),
        # a decode step's slots: 256 requests, some ended, a page needed now and then
        _slots("slots_decode", 256, 16384, 8, 1, 0, 9),
        # prefill chunks and decode tokens in one step
        _slots("slots_mixed", 60, 65536, 8, 2048, 4, 2, padded=7),
    ]


_MOST_BYTES = 5.0e9    # no drawn case costs more than the largest listed one
_MOST_PADDED = 3.2e6   # tokens of the padded gather of the plain form


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    heads = lambda: rng.choice([(32, 8), (32, 8), (32, 4), (4, 1), (8, 2), (28, 4), (8, 8), (16, 1)])  # noqa: E731
    dim = lambda: rng.choice([64, 128, 128])  # noqa: E731
    layout = lambda: rng.choice(["token_major", "transposed"])  # noqa: E731
    while True:
        kind = rng.choice(["decode", "decode", "append", "slots"])
        shape = rng.randrange(1 << 20)
        if kind == "decode":
            batch, longest = spread(1, 256), spread(1, 131072)
            h = heads()
            sparse = rng.random() < 0.3
            ratio = h[0] // h[1]
            group = rng.choice([g for g in range(1, ratio + 1) if ratio % g == 0 and g * 4 >= ratio]) if sparse else ratio
            c = _decode(None, batch, rng.randint(1, longest), longest, h, dim(), layout(),
                        round(rng.uniform(0.03, 0.6), 3) if sparse else 1.0, group,
                        rng.randint(0, batch // 4), 0, shape)
            if batch * longest * h[1] > _MOST_PADDED * 8:
                continue
        elif kind == "append":
            h, d = heads(), dim()
            c = _append(None, spread(1, 64), spread(1, 4096), spread(1, 131072), h, d, layout(),
                        rng.choice([d, d, d // 2]), rng.choice([1, 1, 2, 3, 4]), rng.random() < 0.3,
                        rng.choice([0, 0, rng.randint(1, 9)]), shape)
            if c["requests"] * c["tokens"] > 16384:
                continue
        else:
            batch = spread(1, 2048)
            chunk, chunks = spread(1, 4096), rng.randint(0, min(batch, 6))
            c = _slots(None, batch, spread(64, 65536), rng.choice([1, 2, 4, 8]), chunk, chunks,
                       rng.randint(0, batch - chunks) // 8, rng.choice([0, rng.randint(1, 50)]), shape)
            if batch * c["longest"] * c["kv_heads"] > 3e8:
                continue
        if work(c)["bytes"] <= _MOST_BYTES:
            return c


# ---------------------------------------------------------------------------
# sizes that follow from a case alone
# ---------------------------------------------------------------------------
def _lens(case):
    rng = random.Random(case["shape"])
    if case["kind"] == "decode":
        lo, hi = math.log(case["shortest"]), math.log(case["longest"])
        lens = [int(round(math.exp(rng.uniform(lo, hi)))) for _ in range(case["batch"])]
        lens[0] = case["longest"]
        for i in rng.sample(range(1, case["batch"]), min(case["idle"], case["batch"] - 1)):
            lens[i] = 0
        return lens
    n = case["requests"] if case["kind"] == "append" else case["batch"]
    lens = [int(round(math.exp(rng.uniform(0.0, math.log(case["longest"]))))) for _ in range(n)]
    if case["kind"] == "append":   # some requests start with this call, at a page's start
        lens = [0 if rng.random() < 0.1 else x for x in lens]
    return lens


def _new(case):
    """slots: the tokens that every request adds, and which requests have ended."""
    rng = random.Random(case["shape"] + 1)
    order = rng.sample(range(case["batch"]), case["batch"])
    new, ended = [1] * case["batch"], [0] * case["batch"]
    for i in order[:case["chunks"]]:
        new[i] = case["chunk"]
    for i in order[case["chunks"]:case["chunks"] + case["ended"]]:
        new[i], ended[i] = 0, 1
    return new, ended


def _blocks(n):
    return -(-n // PAGE)


def _counts(case):
    """decode over tables: how many blocks of each request a table row lists."""
    return [min(_blocks(n), max(1, math.ceil(case["density"] * _blocks(n)))) if n else 0 for n in _lens(case)]


def work(case):
    if case["kind"] == "decode":
        lens = _lens(case)
        rows = case["q_heads"] // case["group"]   # table rows of one request
        if case["density"] < 1:   # the last block is listed and may be partly filled
            tokens = [min(n, c * PAGE - (-n) % PAGE) for n, c in zip(lens, _counts(case))]
        else:
            rows, tokens = case["kv_heads"], lens
        kv = rows * sum(tokens) * case["dim"] * 2 * 2
        # page ids (and table entries), queries, outputs, lse
        ids = rows * sum(_blocks(n) for n in tokens) * (8 if case["density"] < 1 else 4)
        io = case["batch"] * case["q_heads"] * (case["dim"] * 4 + 4)
        return {"bytes": kv + ids + io, "flops": 4 * case["dim"] * (case["q_heads"] // rows) * rows * sum(tokens)}
    if case["kind"] == "append":
        t = case["requests"] * case["tokens"]
        rows = t + case["padded"]
        moved = 2 * 2 * case["dim"] * (rows * case["q_heads"] + 2 * t * case["kv_heads"])
        return {"bytes": moved + rows * (4 * case["axes"] + 8 * case["kv_heads"]),
                "flops": 3 * rows * (case["q_heads"] + case["kv_heads"]) * case["rotary"]}
    new, ended = _new(case)
    lens, h = _lens(case), case["kv_heads"]
    t = sum(new) + case["padded"]
    back = sum(_blocks(n) * h for n, e in zip(lens, ended) if e)   # read from the table, written to the list
    got = sum((_blocks(n + m) - _blocks(n)) * h for n, m, e in zip(lens, new, ended) if not e)
    return {"bytes": 8 * back + 8 * got + t * (8 * h + 4) + 28 * case["batch"], "flops": 0}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEVICE)


def _deal_pages(blocks, kv_heads, max_blocks, spare, g):
    """A page table whose requests hold blocks[b] blocks of random pages, -1 elsewhere; the
    pages that no request holds; the number of pages."""
    held = sum(blocks) * kv_heads
    pages = held + spare
    order = torch.randperm(pages, generator=g, device=DEVICE).to(torch.int32)
    table = torch.full((len(blocks), max_blocks, kv_heads), -1, dtype=torch.int32, device=DEVICE)
    listed_ = torch.arange(max_blocks, device=DEVICE)[None, :] < torch.tensor(blocks, device=DEVICE)[:, None]
    table[listed_] = order[:held].view(-1, kv_heads)
    return table.transpose(1, 2).contiguous(), order[held:].contiguous(), pages


def _randn(shape, g, scale=1.0):
    x = torch.randn(shape, generator=g, device=DEVICE, dtype=torch.bfloat16)
    return x if scale == 1.0 else x.mul_(scale)


def _pools(pages, case, g):
    k, v = _randn((pages, PAGE, case["dim"]), g), _randn((pages, PAGE, case["dim"]), g)
    return k, (v.view(pages, case["dim"], PAGE) if case["layout"] == "transposed" else v)


def _prepare_decode(case, seed):
    g = _generator(seed)
    lens, B, H = _lens(case), case["batch"], case["kv_heads"]
    blocks = [_blocks(n) for n in lens]
    max_blocks = max(max(blocks), case["table_blocks"])
    table, _, pages = _deal_pages(blocks, H, max_blocks, 1, g)
    s = dict(kind="decode", case=case, page_table=table, kv_len=_ints(lens), pages=pages,
             max_blocks=max_blocks, scale=case["dim"] ** -0.5, tables=None)
    s["k_pool"], s["v_pool"] = _pools(pages, case, g)
    # scores of standard deviation 2: some keys matter more than others
    s["q"] = _randn((B, case["q_heads"], case["dim"]), g, 2.0)
    if case["density"] < 1:   # every row its own random blocks, the last one among them, ascending
        G = case["q_heads"] // case["group"]
        count, rows = _counts(case), []
        for b in range(B):
            for _ in range(G):
                if not blocks[b]:
                    continue
                pick = torch.randperm(blocks[b] - 1, generator=g, device=DEVICE)[:count[b] - 1]
                last = torch.full((1,), blocks[b] - 1, dtype=pick.dtype, device=DEVICE)
                rows.append(torch.cat([pick.sort().values, last]).to(torch.int32))
        indptr = torch.zeros(B * G + 1, dtype=torch.int64)
        indptr[1:] = torch.tensor([count[b] for b in range(B) for _ in range(G)]).cumsum(0)
        indices = torch.zeros(B * G * max_blocks, dtype=torch.int32, device=DEVICE)
        flat = torch.cat(rows)
        indices[:flat.numel()] = flat
        s["tables"] = (indptr.to(torch.int32).to(DEVICE), indices)
        s["most"] = max(count)
    return s


def _prepare_append(case, seed):
    g = _generator(seed)
    lens, H, T = _lens(case), case["kv_heads"], case["tokens"]
    n = case["requests"]
    blocks = [_blocks(x + T) for x in lens]
    # only the pages that the new tokens are written to are held here: a pool of that size
    first = [x // PAGE for x in lens]
    table, _, pages = _deal_pages([e - f for e, f in zip(blocks, first)], H, max(e - f for e, f in zip(blocks, first)), 1, g)
    pos = torch.tensor(lens, device=DEVICE)[:, None] + torch.arange(T, device=DEVICE)[None, :]
    j = pos // PAGE - torch.tensor(first, device=DEVICE)[:, None]
    page = table.gather(2, j[:, None, :].expand(n, H, T)).long()
    slots = (page * PAGE + pos[:, None, :] % PAGE).permute(0, 2, 1).reshape(n * T, H)
    rows = n * T + case["padded"]
    slot_map = torch.full((rows, H), -1, dtype=torch.int64, device=DEVICE)
    slot_map[:n * T] = slots
    # axis 0 is the token's place in its request; a quarter of the tokens are an image's, whose
    # places on the further axes are a row and a column of it
    positions = torch.zeros((case["axes"], rows), dtype=torch.int32, device=DEVICE)
    positions[:, :n * T] = pos.reshape(1, -1)
    if case["axes"] > 1:
        image = torch.rand(rows, generator=g, device=DEVICE) < 0.25
        places = torch.randint(0, 64, (case["axes"], rows), generator=g, device=DEVICE, dtype=torch.int32)
        positions += places * image
    half = case["rotary"] // 2
    inv_freq = (ROPE_BASE ** (-torch.arange(half, device=DEVICE, dtype=torch.float64) / half)).float()
    s = dict(kind="append", case=case, slot_map=slot_map, positions=positions, inv_freq=inv_freq,
             pages=pages, max_blocks=table.shape[2],
             pair_axis=[i * case["axes"] // half for i in range(half)])
    # queries, keys and values leave the projection in one tensor
    Hq, D = case["q_heads"], case["dim"]
    qkv = _randn((rows, Hq + 2 * H, D), g)
    s["q"], s["k"], s["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
    s["k_pool"], s["v_pool"] = _pools(pages, case, g)
    return s


def _prepare_slots(case, seed):
    g = _generator(seed)
    lens, (new, ended) = _lens(case), _new(case)
    H = case["kv_heads"]
    most = max(_blocks(n + m) for n, m in zip(lens, new))
    need = sum((_blocks(n + m) - _blocks(n)) * H for n, m in zip(lens, new))
    table, free, pages = _deal_pages([_blocks(n) for n in lens], H, most, need + 64, g)
    free_pages = torch.full((pages,), -1, dtype=torch.int32, device=DEVICE)
    free_pages[:free.numel()] = free
    return dict(kind="slots", case=case, page_table=table, free_pages=free_pages, pages=pages,
                max_blocks=most, free_count=_ints([free.numel()]), seq_len=_ints(lens),
                new_len=_ints(new), ended=_ints(ended) if case["ended"] else None,
                tokens=sum(new) + case["padded"])


def prepare(case, seed):
    s = {"decode": _prepare_decode, "append": _prepare_append, "slots": _prepare_slots}[case["kind"]](case, seed)
    if own:   # the sizes' descriptors, and the workspace, which a program keeps from step to step
        _own_handles(s)
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(s):
    return {"decode": _run_decode, "append": _run_append, "slots": _run_slots}[s["kind"]](s)


def _own_handles(s):
    import paper_2605_16839_amd as ca

    c = s["case"]
    s["cache"] = ca.Cache(batch=s["page_table"].shape[0] if "page_table" in s else 1,
                          num_q_heads=c.get("q_heads", c["kv_heads"]), num_kv_heads=c["kv_heads"],
                          head_dim=c.get("dim", 128), max_kv_blocks=s["max_blocks"], num_pages=s["pages"],
                          v_layout=ca.V_TRANSPOSED if c.get("layout") == "transposed" else ca.V_TOKEN_MAJOR)
    if s["kind"] == "decode":
        s["ws"] = torch.empty(ca.decode_workspace_bytes(s["cache"], c["group"]), dtype=torch.uint8, device=DEVICE)
    if s["kind"] == "append":
        s["rotary"] = ca.Rotary(s["inv_freq"], interleaved=c["interleaved"], num_axes=c["axes"],
                                pair_axis=s["pair_axis"])


def _run_decode(s):
    c = s["case"]
    if own:
        import paper_2605_16839_amd as ca

        lse = torch.empty(s["q"].shape[:2], dtype=torch.float32, device=DEVICE)
        out, _ = ca.decode_attention(s["cache"], s["q"], (s["k_pool"], s["v_pool"]), s["page_table"],
                                     s["kv_len"], s["scale"], tables=s["tables"], group_size=c["group"],
                                     lse=lse, ws=s["ws"])
        return {"out": out, "lse": lse}
    B, Hq, D = s["q"].shape
    H, gs = c["kv_heads"], c["group"]
    G = Hq // gs
    if s["tables"] is None:   # G == H: every block of the request
        block = torch.arange(s["page_table"].shape[2], device=DEVICE)[:int(_blocks(c["longest"]))].expand(B, G, -1)
        live = block < ((s["kv_len"] + PAGE - 1) // PAGE)[:, None, None]
    else:
        indptr, indices = s["tables"]
        first, count = indptr[:-1].view(B, G, 1).long(), indptr.diff().view(B, G, 1)
        at = torch.arange(s["most"], device=DEVICE).expand(B, G, -1)
        live = at < count
        block = indices[torch.where(live, first + at, 0)].long()
    head = torch.arange(G, device=DEVICE) * gs // (Hq // H)   # the KV head of a group
    page = s["page_table"][:, head].gather(2, block)
    page = torch.where(live, page, 0).long()
    seen = live[..., None] & (block[..., None] * PAGE + torch.arange(PAGE, device=DEVICE) < s["kv_len"][:, None, None, None])
    seen = seen.flatten(2)   # [B, G, keys]
    keys = s["k_pool"][page].flatten(2, 3).float()
    score = torch.matmul(s["q"].view(B, G, gs, D).float(), keys.transpose(2, 3)) * s["scale"]
    del keys
    score = score.masked_fill(~seen[:, :, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    weight = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    total = weight.sum(-1, keepdim=True)
    values = s["v_pool"][page]
    values = (values.transpose(3, 4) if c["layout"] == "transposed" else values).flatten(2, 3).float()
    values = torch.where(seen[..., None], values, 0.0)
    out = torch.matmul(weight, values) / torch.where(total == 0, 1.0, total)
    return {"out": out.view(B, Hq, D).to(torch.bfloat16), "lse": (top + torch.log(total)).view(B, Hq)}


def _rotated(x, angle_cos, angle_sin, rotary, interleaved):
    """x [rows, heads, D], the cosines and sines [rows, 1, rotary / 2]."""
    part, rest = x[..., :rotary], x[..., rotary:]
    a, b = (part[..., 0::2], part[..., 1::2]) if interleaved else part.chunk(2, -1)
    u, w = a * angle_cos - b * angle_sin, b * angle_cos + a * angle_sin
    part = torch.stack([u, w], -1).flatten(-2) if interleaved else torch.cat([u, w], -1)
    return torch.cat([part, rest], -1)


def _angles(s):
    """[rows, 1, rotary / 2] in 64 bits: far positions lose their place in 32."""
    place = s["positions"][torch.tensor(s["pair_axis"], device=DEVICE)].t().double()
    return (place * s["inv_freq"].double())[:, None]


def _run_append(s):
    c = s["case"]
    if own:
        import paper_2605_16839_amd as ca

        q = ca.rotary_append(s["cache"], s["rotary"], s["q"], s["k"], s["v"], s["positions"], s["slot_map"],
                             (s["k_pool"], s["v_pool"]))
        return {"q": q, "k_pool": s["k_pool"], "v_pool": s["v_pool"]}
    angle = _angles(s)
    cos, sin = angle.cos().float(), angle.sin().float()
    q = _rotated(s["q"].float(), cos, sin, c["rotary"], c["interleaved"]).to(torch.bfloat16)
    k = _rotated(s["k"].float(), cos, sin, c["rotary"], c["interleaved"]).to(torch.bfloat16)
    row, head = torch.where(s["slot_map"] >= 0)
    slot = s["slot_map"][row, head]
    s["k_pool"][slot // PAGE, slot % PAGE] = k[row, head]
    if c["layout"] == "transposed":
        s["v_pool"][slot // PAGE, :, slot % PAGE] = s["v"][row, head]
    else:
        s["v_pool"][slot // PAGE, slot % PAGE] = s["v"][row, head]
    return {"q": q, "k_pool": s["k_pool"], "v_pool": s["v_pool"]}


def _run_slots(s):
    if own:
        import paper_2605_16839_amd as ca

        seq_len, free_count = s["seq_len"], s["free_count"]
        if s["ended"] is not None:
            seq_len, free_count = ca.release_pages(s["cache"], s["ended"], seq_len, s["page_table"],
                                                   s["free_pages"], free_count)
        a = ca.assign_slots(s["cache"], s["new_len"], s["tokens"], seq_len, s["page_table"], s["free_pages"],
                            free_count)
        return {"slot_map": a["slot_map"], "positions": a["positions"], "token_indptr": a["token_indptr"],
                "granted": a["granted"], "seq_len": a["seq_len"], "free_count": a["free_count"],
                "page_table": s["page_table"], "free_pages": s["free_pages"]}
    table, free_pages = s["page_table"], s["free_pages"]
    B, H, most = table.shape
    old, count = s["seq_len"].long(), s["free_count"].long()
    if s["ended"] is not None:   # their pages go behind the free ones, request by request, block by block
        held = torch.where(s["ended"] != 0, (old + PAGE - 1) // PAGE, 0)
        back = torch.arange(most, device=DEVICE)[None, :] < held[:, None]
        pages = table.transpose(1, 2)[back].flatten()
        free_pages[count + torch.arange(pages.numel(), device=DEVICE)] = pages
        old = torch.where(s["ended"] != 0, 0, old)
        count = count + pages.numel()
    new = s["new_len"].long()
    end = new.cumsum(0)
    start = end - new
    had, has = (old + PAGE - 1) // PAGE, (old + new + PAGE - 1) // PAGE
    fits = (has <= most) & (end <= s["tokens"])
    need = torch.where(fits, (has - had) * H, 0)
    taken = need.cumsum(0)
    fits = fits & ((need == 0) | (taken <= count))
    first = taken - need   # a request's pages follow those of the requests before it, from the list's end down
    granted = torch.where(fits, new, 0)
    t = torch.arange(s["tokens"], device=DEVICE)
    b = torch.searchsorted(end, t, right=True)
    real = b < B
    b = torch.where(real, b, 0)
    real = real & fits[b]
    pos = torch.where(real, old[b] + t - start[b], 0)
    j = pos // PAGE
    fresh = real & (j >= had[b])
    h = torch.arange(H, device=DEVICE)
    place = count - 1 - (first[b] + (j - had[b]) * H)[:, None] - h
    page = torch.where(fresh[:, None], free_pages[torch.where(fresh[:, None], place, 0)], table[b[:, None], h, j[:, None]])
    opens = torch.where(fresh & (pos % PAGE == 0))[0]
    table[b[opens, None], h, j[opens, None]] = page[opens]
    ok = real[:, None] & (page >= 0) & (page < s["pages"])
    slot_map = torch.where(ok, page.long() * PAGE + (pos % PAGE)[:, None], -1)
    left = count - torch.where(fits, need, 0).sum()
    indptr = torch.cat([start.new_zeros(1), end]).clamp(max=s["tokens"])
    i32 = torch.int32
    return {"slot_map": slot_map, "positions": pos.to(i32), "token_indptr": indptr.to(i32),
            "granted": granted.to(i32), "seq_len": (old + granted).to(i32), "free_count": left.to(i32),
            "page_table": table, "free_pages": free_pages}


# ---------------------------------------------------------------------------
# the same from the definitions, in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    if case["kind"] == "slots":
        return None   # whole numbers only
    s = {"decode": _prepare_decode, "append": _prepare_append}[case["kind"]](case, seed)
    return _exact_decode(case, s) if case["kind"] == "decode" else _exact_append(case, s)


def _exact_decode(case, s):
    Hq, H, D = case["q_heads"], case["kv_heads"], case["dim"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device=DEVICE)
    ends = s["tables"][0].tolist() if s["tables"] else None
    for b, n in enumerate(_lens(case)):
        for g in range(Hq // case["group"]):
            if n == 0:
                continue
            heads = slice(g * case["group"], (g + 1) * case["group"])
            kvh = g * case["group"] // (Hq // H)
            if ends:
                r = b * (Hq // case["group"]) + g
                listed_ = s["tables"][1][ends[r]:ends[r + 1]].long()
            else:
                listed_ = torch.arange(_blocks(n), device=DEVICE)
            pages = s["page_table"][b, kvh, listed_].long()
            k, v = s["k_pool"][pages].double(), s["v_pool"][pages].double()
            if case["layout"] == "transposed":
                v = v.transpose(1, 2)
            keep = ((listed_ * PAGE)[:, None] + torch.arange(PAGE, device=DEVICE)).flatten() < n
            k, v = k.reshape(-1, D)[keep], v.reshape(-1, D)[keep]
            x = s["q"][b, heads].double() @ k.t() * s["scale"]
            z = torch.logsumexp(x, -1)
            lse[b, heads] = z
            out[b, heads] = torch.exp(x - z[:, None]) @ v
    return {"out": out, "lse": lse}


def _exact_append(case, s):
    R, rows = case["rotary"], s["q"].shape[0]
    turned = []
    where = s["positions"].double()
    axis = torch.tensor(s["pair_axis"], device=DEVICE)
    for x in (s["q"], s["k"]):
        y = x.double().clone()
        for i in range(R // 2):   # pair i turns by its axis' place times its frequency
            angle = where[axis[i]] * s["inv_freq"][i].double()
            at = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + R // 2)
            z = torch.complex(x[..., at[0]].double(), x[..., at[1]].double()) * torch.polar(torch.ones_like(angle), angle).view(rows, 1)
            y[..., at[0]], y[..., at[1]] = z.real, z.imag
        turned.append(y)
    pool = s["k_pool"].double().view(-1, case["dim"])
    for h in range(case["kv_heads"]):
        kept = s["slot_map"][:, h] >= 0
        pool[s["slot_map"][kept, h]] = turned[1][kept, h]
    return {"q": turned[0], "k_pool": pool.view(s["k_pool"].shape), "v_pool": None}
