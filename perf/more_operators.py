"""Requests that share pages of the KV cache, and normalised heads, as cases that can be timed and compared.

Several answers of one prompt, beams, and requests behind one system prompt hold the same
pages.  ``sharing.fork_requests`` makes rows of the page table forks of others and gives
back what no one holds any more, ``sharing.compact_pages`` moves the pages in use to the
lowest ids, and ``sharing.prefix_decode_attention`` reads a shared prefix once for all of its
requests.  ``rotary_append`` with a ``HeadNorm`` normalises every head of queries and
keys before it turns them.

Kinds of cases:
  prefix   prefix_decode_attention of one step
  fork     fork_requests
  compact  compact_pages
  norm     rotary_append with norms
"""
import math
import random

import torch

own = False   # set from outside: True runs this package's kernels, False the plain forms

PAGE = 64
DEVICE = "cuda"
ROPE_BASE = 500000.0   # of the LLaMA-3.1 layer that the workloads are shaped after
EPS = 1e-5


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------
def _named(name, case):
    return dict(name=name, **case) if name else case


def _prefix(name, batch, shares, shortest, longest, least, most, heads, dim, layout, idle=0, alone=0, shape=1):
    """batch requests: idle of them empty, alone of them in no share, the others dealt to shares whose
    prefixes have shortest to longest tokens; each has least to most tokens of its own behind its prefix."""
    return _named(name, dict(kind="prefix", batch=batch, shares=shares, shortest=shortest, longest=longest, least=least,
                             most=most, q_heads=heads[0], kv_heads=heads[1], dim=dim, layout=layout, idle=idle,
                             alone=alone, shape=shape))


def _fork(name, groups, width, shortest, longest, kv_heads, dim, layout, moves, cut=False, shape=1):
    """groups of width rows.  moves "first": the first row of each holds a prompt, the others become its
    forks; "beams": all rows are forks of one prompt with a tail of their own, and each goes on from a row
    drawn from its group (some rows end, some keep theirs); cut: up to a length drawn, not to the end."""
    return _named(name, dict(kind="fork", groups=groups, width=width, shortest=shortest, longest=longest,
                             kv_heads=kv_heads, dim=dim, layout=layout, moves=moves, cut=cut, shape=shape))


def _compact(name, batch, shortest, longest, kv_heads, dim, spare, shape=1):
    """batch requests of shortest to longest tokens whose pages lie anywhere in a pool with spare times as
    many free pages; every fourth request shares its first half with the request before it."""
    return _named(name, dict(kind="compact", batch=batch, shortest=shortest, longest=longest, kv_heads=kv_heads,
                             dim=dim, spare=spare, shape=shape))


def _norm(name, requests, tokens, longest, heads, dim, layout, rotary, axes=1, interleaved=False, padded=0,
          wide=False, offset=False, shape=1):
    """tokens new tokens of each request, whose cached lengths go up to longest; padded more rows belong to no
    request; weights in 32 bits (wide) or bf16, stored less 1 (offset) or as they are."""
    return _named(name, dict(kind="norm", requests=requests, tokens=tokens, longest=longest, q_heads=heads[0],
                             kv_heads=heads[1], dim=dim, layout=layout, rotary=rotary, axes=axes,
                             interleaved=interleaved, padded=padded, wide=wide, offset=offset, shape=shape))


def listed():
    return [
        # the smallest call: three answers of a short prompt on a small model, where latency counts
        _prefix("prefix_small", 3, 1, 700, 700, 1, 90, (4, 1), 64, "token_major"),
        # 64 samples of one long prompt
        _prefix("prefix_samples", 64, 1, 32768, 32768, 1, 2048, (32, 8), 128, "token_major"),
        # several system prompts of different lengths, some requests behind none, captured for 96 with 7 rows idle
        _prefix("prefix_agents", 96, 6, 1500, 16000, 64, 6000, (32, 8), 128, "token_major", idle=7, alone=5),
        # questions about one long document, grouped queries of 8 heads per KV head, transposed V pages
        _prefix("prefix_document", 16, 1, 60001, 60001, 30, 3000, (32, 4), 128, "transposed"),
        # the largest call: a full batch behind a prefix of almost 128K tokens
        _prefix("prefix_large", 128, 1, 126976, 126976, 16, 4096, (32, 8), 128, "token_major"),
        # a prompt of 32K tokens becomes 64 requests
        _fork("fork_samples", 1, 64, 32741, 32741, 8, 128, "token_major", "first"),
        # beams of 16 prompts are reordered: every step of a beam search
        _fork("fork_beams", 16, 4, 500, 9000, 8, 128, "transposed", "beams"),
        # a small pool
        _compact("compact_small", 5, 100, 2000, 2, 64, 0.7),
        # half of a large pool is free after a burst of requests
        _compact("compact_large", 48, 2000, 20000, 8, 128, 1.0),
        # one decode step's tokens, captured for 64 with 5 rows idle
        _norm("norm_decode", 59, 1, 32768, (32, 8), 128, "token_major", 128, padded=5),
        # four prefill chunks of 2048 tokens
        _norm("norm_chunks", 4, 2048, 126976, (32, 8), 128, "token_major", 128),
        # a prompt's remainder with image tokens: positions of three axes, half of a head turned, transposed V pages
        _norm("norm_axes", 3, 1451, 50001, (28, 4), 128, "transposed", 64, axes=3, wide=True, offset=True),
    ]


_MOST_COST = 2.0e9     # bytes, or flops / 100: no drawn case costs more than the largest listed one
_MOST_PADDED = 1.5e9   # elements of the padded tensors of the plain forms


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 100)


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    heads = lambda: rng.choice([(32, 8), (32, 8), (32, 4), (4, 1), (8, 2), (28, 4), (8, 8), (16, 1)])  # noqa: E731
    dim = lambda: rng.choice([64, 128, 128])  # noqa: E731
    layout = lambda: rng.choice(["token_major", "transposed"])  # noqa: E731
    while True:
        kind = rng.choice(["prefix", "prefix", "fork", "compact", "norm"])
        shape = rng.randrange(1 << 20)
        if kind == "prefix":
            batch = spread(1, 256)
            longest, most = spread(1, 126976), spread(1, 8192)
            c = _prefix(None, batch, rng.randint(1, min(8, batch)), rng.randint(1, longest), longest,
                        rng.randint(1, most), most, heads(), dim(), layout(), rng.randint(0, batch // 4),
                        rng.randint(0, batch // 4), shape)
            keys = c["kv_heads"] * (c["shares"] * (longest + PAGE) + batch * (most + PAGE))
            scores = c["q_heads"] * batch * (c["shares"] * (longest + PAGE) + most + PAGE)
            if keys * c["dim"] > _MOST_PADDED or scores > _MOST_PADDED:
                continue
        elif kind == "fork":
            longest = spread(1, 65536)
            c = _fork(None, spread(1, 32), spread(1, 32), rng.randint(1, longest), longest, rng.choice([1, 2, 4, 8]),
                      dim(), layout(), rng.choice(["first", "beams", "beams"]), rng.random() < 0.3, shape)
            if c["groups"] * (longest + 320 * c["width"]) * c["kv_heads"] > 4e6:
                continue
        elif kind == "compact":
            longest = spread(1, 30000)
            c = _compact(None, spread(1, 64), rng.randint(1, longest), longest, rng.choice([1, 2, 4, 8]), dim(),
                         round(rng.uniform(0.05, 2.0), 2), shape)
            if c["batch"] * longest * c["kv_heads"] * (1 + c["spare"]) > 1e7:
                continue
        else:
            h, d = heads(), dim()
            c = _norm(None, spread(1, 64), spread(1, 4096), spread(1, 131072), h, d, layout(),
                      rng.choice([d, d, d // 2, 0]), rng.choice([1, 1, 2, 3, 4]), rng.random() < 0.3,
                      rng.choice([0, 0, rng.randint(1, 9)]), rng.random() < 0.5, rng.random() < 0.3, shape)
            if c["requests"] * c["tokens"] > 16384:
                continue
        if _cost(c) <= _MOST_COST:
            return c


# ---------------------------------------------------------------------------
# sizes that follow from a case alone
# ---------------------------------------------------------------------------
def _blocks(n):
    return -(-n // PAGE)


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _prefix_plan(case):
    """(tokens of each share's prefix, share of each request, tokens of each request)."""
    rng = random.Random(case["shape"])
    prefix = [_spread(rng, case["shortest"], case["longest"]) for _ in range(case["shares"])]
    prefix[0] = case["longest"]
    B = case["batch"]
    share = [rng.randrange(case["shares"]) for _ in range(B)]
    mine = [_spread(rng, case["least"], case["most"]) for _ in range(B)]
    order = rng.sample(range(B), B)
    lens = [prefix[s] + n for s, n in zip(share, mine)]
    for b in order[:case["idle"]]:      # still named in its share, with nothing in its row
        lens[b] = 0
    for b in order[case["idle"]:case["idle"] + case["alone"]]:
        share[b], lens[b] = -1, mine[b]
    return prefix, share, lens


def _fork_plan(case):
    """Of every row: its cached tokens, the tokens that it shares with its group's first row (whole pages of
    them), the row that it goes on from (-1: it ends), the tokens to keep (None: all)."""
    rng = random.Random(case["shape"])
    W = case["width"]
    lens, common, parent = [], [], []
    for g in range(case["groups"]):
        prompt = _spread(rng, case["shortest"], case["longest"])
        if case["moves"] == "first":
            lens += [prompt] + [0] * (W - 1)
            common += [0] * W
            parent += [g * W] * W
        else:
            lens += [prompt + rng.randint(0, 256) for _ in range(W)]
            common += [0] + [prompt // PAGE * PAGE] * (W - 1)
            parent += [rng.choice([g * W + i] * 2 + [g * W + rng.randrange(W)] * 5 + [-1]) for i in range(W)]
    keep = [rng.randint(0, case["longest"] + 256) for _ in lens] if case["cut"] else None
    return lens, common, parent, keep


def _compact_plan(case):
    """Of every request: its tokens and the blocks that it shares with the request before it."""
    rng = random.Random(case["shape"])
    lens = [_spread(rng, case["shortest"], case["longest"]) for _ in range(case["batch"])]
    shared = [min(lens[b] // PAGE, lens[b - 1] // PAGE) // 2 if b % 4 == 1 else 0 for b in range(len(lens))]
    held = (sum(_blocks(n) for n in lens) - sum(shared)) * case["kv_heads"]
    pages = held + max(1, int(held * case["spare"]))
    return lens, shared, held, pages


def _norm_lens(case):
    rng = random.Random(case["shape"])
    lens = [_spread(rng, 1, case["longest"]) for _ in range(case["requests"])]
    return [0 if rng.random() < 0.1 else n for n in lens]   # some start with this call, at a page's start


def _kept(lens, parent, keep):
    """Tokens of every row after the call, and whether the row is another than before."""
    new = [0 if p < 0 else lens[p] if keep is None else min(lens[p], keep[b]) for b, p in enumerate(parent)]
    return new, [p != b or new[b] != lens[b] for b, p in enumerate(parent)]


def _copies(new, parent):
    """Rows whose last page is part-filled and someone else's too (shared prefixes are whole pages)."""
    full, count = [n // PAGE for n in new], 0
    for b, p in enumerate(parent):
        if p < 0 or new[b] % PAGE == 0:
            continue
        for o, po in enumerate(parent):
            if o != b and po == p and (full[o] > full[b] or (full[o] == full[b] and new[o] % PAGE
                                                             and (o == p or (o < b and b != p)))):
                count += 1
                break
    return count


def work(case):
    kind, D = case["kind"], case["dim"]
    page_bytes = 2 * PAGE * D * 2   # of K and V
    if kind == "prefix":
        prefix, share, lens = _prefix_plan(case)
        H, Hq = case["kv_heads"], case["q_heads"]
        whole = [n // PAGE * PAGE for n in prefix]
        used = {s for s, n in zip(share, lens) if s >= 0 and n}
        tokens = sum(whole[s] for s in used) + sum(n - (whole[s] if s >= 0 and n else 0) for s, n in zip(share, lens))
        ids = H * 4 * sum(_blocks(n) for n in lens)
        io = case["batch"] * Hq * (D * 4 + 4)
        return {"bytes": tokens * H * D * 4 + ids + io, "flops": 4 * D * Hq * sum(lens)}
    if kind == "fork":
        lens, _, parent, keep = _fork_plan(case)
        new, changed = _kept(lens, parent, keep)
        H = case["kv_heads"]
        entries = sum(_blocks(n) for n in new) * H
        counted = sum(_blocks(n) + _blocks(m) for n, m, c in zip(new, lens, changed) if c) * H
        return {"bytes": 8 * entries + 8 * counted + 2 * page_bytes * _copies(new, parent) * H + 12 * len(lens), "flops": 0}
    if kind == "compact":
        lens, _, held, pages = _compact_plan(case)
        entries = sum(_blocks(n) for n in lens) * case["kv_heads"]
        moved = held * (pages - held) // pages   # as many free ids as that are below the pages' number, on average
        return {"bytes": 2 * page_bytes * moved + 8 * entries + 12 * pages + 8 * (pages - held), "flops": 0}
    t = case["requests"] * case["tokens"]
    rows = t + case["padded"]
    moved = 2 * 2 * D * (rows * case["q_heads"] + 2 * t * case["kv_heads"])
    return {"bytes": moved + rows * (4 * case["axes"] + 8 * case["kv_heads"]),
            "flops": rows * (case["q_heads"] + case["kv_heads"]) * (3 * case["rotary"] + 4 * D)}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEVICE)


def _randn(shape, g, scale=1.0):
    x = torch.randn(shape, generator=g, device=DEVICE, dtype=torch.bfloat16)
    return x if scale == 1.0 else x.mul_(scale)


def _pools(pages, case, g):
    k, v = _randn((pages, PAGE, case["dim"]), g), _randn((pages, PAGE, case["dim"]), g)
    return k, (v.view(pages, case["dim"], PAGE) if case.get("layout") == "transposed" else v)


def _deal(blocks, first, kv_heads, max_blocks, g, spare):
    """A page table whose row b holds random pages of its own in blocks first[b] .. blocks[b] - 1 (-1
    elsewhere), the pages that no row holds, and the number of pages."""
    own_blocks = [n - f for n, f in zip(blocks, first)]
    held = sum(own_blocks) * kv_heads
    order = torch.randperm(held + spare, generator=g, device=DEVICE).to(torch.int32)
    table = torch.full((len(blocks), max_blocks, kv_heads), -1, dtype=torch.int32, device=DEVICE)
    at = torch.arange(max_blocks, device=DEVICE)[None, :]
    mine = (at < torch.tensor(blocks, device=DEVICE)[:, None]) & (at >= torch.tensor(first, device=DEVICE)[:, None])
    table[mine] = order[:held].view(-1, kv_heads)
    return table.transpose(1, 2).contiguous(), order[held:].contiguous(), held + spare


def _prepare_prefix(case, seed):
    g = _generator(seed)
    prefix, share, lens = _prefix_plan(case)
    B, H, S = case["batch"], case["kv_heads"], case["shares"]
    whole = [n // PAGE for n in prefix]
    # rows of the shares' own pages behind the requests' rows, from which the members take theirs
    first = [whole[s] if s >= 0 and n else 0 for s, n in zip(share, lens)]
    blocks = [_blocks(n) for n in lens]
    most = max(max(blocks), 1)
    table, _, pages = _deal(blocks + whole, first + [0] * S, H, max(most, max(whole)), g, 1)
    mark = _ints([s if n else -1 for s, n in zip(share, lens)]).long()
    at = torch.arange(most, device=DEVICE) < _ints(first)[:, None]
    rows = table[B:][mark.clamp(min=0)][:, :, :most]
    page_table = torch.where(at[:, None, :], rows, table[:B, :, :most]).contiguous()
    s = dict(kind="prefix", case=case, page_table=page_table, kv_len=_ints(lens), share=_ints(share),
             share_len=_ints(prefix), pages=pages, max_blocks=most, scale=case["dim"] ** -0.5)
    s["k_pool"], s["v_pool"] = _pools(pages, case, g)
    # scores of standard deviation 2: some keys matter more than others
    s["q"] = _randn((B, case["q_heads"], case["dim"]), g, 2.0)
    return s


def _prepare_fork(case, seed):
    g = _generator(seed)
    lens, common, parent, keep = _fork_plan(case)
    H, W = case["kv_heads"], case["width"]
    blocks, first = [_blocks(n) for n in lens], [n // PAGE for n in common]
    most = max(max(blocks), 1) + 2
    table, free, pages = _deal(blocks, first, H, most, g, H * len(lens) + 40)
    row = torch.arange(len(lens), device=DEVICE)
    at = torch.arange(most, device=DEVICE) < _ints(first)[:, None]
    table = torch.where(at[:, None, :], table[row // W * W], table).contiguous()
    held = torch.arange(most, device=DEVICE) < _ints(blocks)[:, None]
    ids = table[held[:, None, :].expand_as(table)].long()
    page_shares = torch.bincount(ids, minlength=pages).sub(1).clamp(min=0).to(torch.int32)
    free_pages = torch.full((pages,), -1, dtype=torch.int32, device=DEVICE)
    free_pages[:free.numel()] = free
    s = dict(kind="fork", case=case, page_table=table, page_shares=page_shares, free_pages=free_pages,
             free_count=_ints([free.numel()]), seq_len=_ints(lens), parent=_ints(parent),
             keep=_ints(keep) if keep else None, pages=pages, max_blocks=most)
    s["k_pool"], s["v_pool"] = _pools(pages, case, g)
    _after(s, ("seq_len", "page_table", "page_shares", "free_pages", "free_count"))
    return s


def _prepare_compact(case, seed):
    g = _generator(seed)
    lens, shared, _, pages = _compact_plan(case)
    H = case["kv_heads"]
    blocks = [_blocks(n) for n in lens]
    most = max(blocks)
    held = (sum(blocks) - sum(shared)) * H
    table, free, _ = _deal(blocks, shared, H, most, g, pages - held)
    at = torch.arange(most, device=DEVICE) < _ints(shared)[:, None]
    table = torch.where(at[:, None, :], table.roll(1, 0), table).contiguous()
    page_shares = torch.zeros(pages, dtype=torch.int32, device=DEVICE)
    page_shares[table[at[:, None, :].expand_as(table)].long()] = 1
    free_pages = torch.full((pages,), -1, dtype=torch.int32, device=DEVICE)
    free_pages[:free.numel()] = free
    s = dict(kind="compact", case=case, page_table=table, page_shares=page_shares, free_pages=free_pages,
             free_count=_ints([free.numel()]), seq_len=_ints(lens), pages=pages, max_blocks=most)
    s["k_pool"], s["v_pool"] = _pools(pages, case, g)
    _after(s, ("page_table", "page_shares", "free_pages", "free_count"))
    s["after"]["new_page"] = torch.full((pages,), -1, dtype=torch.int32, device=DEVICE)
    return s


def _after(s, names):
    """Buffers for the state after the call; entries that a call leaves alone stay -1."""
    s["after"] = {n: torch.full_like(s[n], -1) for n in names}


def _prepare_norm(case, seed):
    g = _generator(seed)
    lens, H, T, n = _norm_lens(case), case["kv_heads"], case["tokens"], case["requests"]
    # only the pages that the new tokens are written to are held here: a pool of that size
    base = [x // PAGE for x in lens]
    blocks = [_blocks(x + T) - f for x, f in zip(lens, base)]
    table, _, pages = _deal(blocks, [0] * n, H, max(blocks), g, 1)
    pos = torch.tensor(lens, device=DEVICE)[:, None] + torch.arange(T, device=DEVICE)[None, :]
    j = pos // PAGE - torch.tensor(base, device=DEVICE)[:, None]
    page = table.gather(2, j[:, None, :].expand(n, H, T)).long()
    slots = (page * PAGE + pos[:, None, :] % PAGE).permute(0, 2, 1).reshape(n * T, H)
    rows, D, Hq = n * T + case["padded"], case["dim"], case["q_heads"]
    slot_map = torch.full((rows, H), -1, dtype=torch.int64, device=DEVICE)
    slot_map[:n * T] = slots
    # axis 0 is the token's place in its request; a quarter of the tokens are an image's, whose
    # places on the further axes are a row and a column of it
    positions = torch.zeros((case["axes"], rows), dtype=torch.int32, device=DEVICE)
    positions[:, :n * T] = pos.reshape(1, -1)
    if case["axes"] > 1:
        image = torch.rand(rows, generator=g, device=DEVICE) < 0.25
        positions += torch.randint(0, 64, (case["axes"], rows), generator=g, device=DEVICE, dtype=torch.int32) * image
    half = case["rotary"] // 2
    s = dict(kind="norm", case=case, slot_map=slot_map, positions=positions, pages=pages, max_blocks=max(blocks),
             inv_freq=(ROPE_BASE ** (-torch.arange(half, device=DEVICE, dtype=torch.float64) / max(half, 1))).float(),
             pair_axis=[i * case["axes"] // max(half, 1) for i in range(half)])
    # queries, keys and values leave the projection in one tensor
    qkv = _randn((rows, Hq + 2 * H, D), g)
    s["q"], s["k"], s["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
    for name in ("q_weight", "k_weight"):   # around 1, as trained ones are
        w = 1.0 + 0.2 * torch.randn(D, generator=g, device=DEVICE) - (1.0 if case["offset"] else 0.0)
        s[name] = w if case["wide"] else w.to(torch.bfloat16)
    s["k_pool"], s["v_pool"] = _pools(pages, case, g)
    return s


_PREPARE = {"prefix": _prepare_prefix, "fork": _prepare_fork, "compact": _prepare_compact, "norm": _prepare_norm}


def prepare(case, seed):
    s = _PREPARE[case["kind"]](case, seed)
    if own:   # the sizes' descriptors, and the workspace, which a program keeps from step to step
        _own_handles(s)
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(s):
    return {"prefix": _run_prefix, "fork": _run_fork, "compact": _run_compact, "norm": _run_norm}[s["kind"]](s)


def _own_handles(s):
    import paper_2605_16839_amd as ca

    c = s["case"]
    s["cache"] = ca.Cache(batch=s["page_table"].shape[0] if "page_table" in s else 1,
                          num_q_heads=c.get("q_heads", c["kv_heads"]), num_kv_heads=c["kv_heads"],
                          head_dim=c["dim"], max_kv_blocks=s["max_blocks"], num_pages=s["pages"],
                          v_layout=ca.V_TRANSPOSED if c.get("layout") == "transposed" else ca.V_TOKEN_MAJOR)
    if s["kind"] == "norm":
        norm = ca.HeadNorm(s["q_weight"], s["k_weight"], eps=EPS, unit_offset=c["offset"])
        s["rotary"] = ca.Rotary(s["inv_freq"] if c["rotary"] else None, interleaved=c["interleaved"],
                                num_axes=c["axes"], pair_axis=s["pair_axis"], norm=norm)
        return
    size = {"prefix": lambda: ca.sharing.prefix_decode_workspace_bytes(s["cache"], c["shares"]),
            "fork": lambda: ca.sharing.fork_workspace_bytes(s["cache"]),
            "compact": lambda: ca.sharing.compact_workspace_bytes(s["cache"])}[s["kind"]]()
    s["ws"] = torch.empty(size, dtype=torch.uint8, device=DEVICE)


def _part(q, keys, values, seen, scale):
    """Unnormalised attention q [.., R, D] over keys [.., N, D]: the largest score, the sum of weights and the
    weighted sum; seen [.., 1 or R, N]."""
    score = torch.matmul(q, keys.transpose(-1, -2)) * scale
    score = score.masked_fill(~seen, -math.inf)
    top = score.amax(-1, keepdim=True)
    weight = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    return top, weight.sum(-1, keepdim=True), torch.matmul(weight, values)


def _pages(s, page, live):
    """Keys and values in 32 bits of pages [.., n]: [.., n * 64, D], 0 where no page is."""
    page = torch.where(live, page, 0).long()
    k, v = s["k_pool"][page].float(), s["v_pool"][page].float()
    v = v.transpose(-1, -2) if s["case"]["layout"] == "transposed" else v
    none = ~live[..., None, None]
    return k.masked_fill(none, 0.0).flatten(-3, -2), v.masked_fill(none, 0.0).flatten(-3, -2)


def _run_prefix(s):
    c = s["case"]
    if own:
        import paper_2605_16839_amd as ca

        lse = torch.empty(s["q"].shape[:2], dtype=torch.float32, device=DEVICE)
        out, _ = ca.sharing.prefix_decode_attention(s["cache"], s["q"], (s["k_pool"], s["v_pool"]), s["page_table"],
                                                    s["kv_len"], s["share"], s["share_len"], s["scale"], lse=lse,
                                                    ws=s["ws"])
        return {"out": out, "lse": lse}
    B, Hq, D = s["q"].shape
    H, S = c["kv_heads"], c["shares"]
    G = Hq // H
    q = s["q"].view(B, H, G, D).float()
    table, lens = s["page_table"], s["kv_len"].long()
    whole = s["share_len"].long() // PAGE
    share = s["share"].long()
    member = (share >= 0) & (lens >= whole[share.clamp(min=0)] * PAGE) & (whole[share.clamp(min=0)] > 0)
    skip = torch.where(member, whole[share.clamp(min=0)], 0)
    # the requests' own pages, padded to the most that one has
    n = int(_blocks(c["most"] + PAGE - 1)) + 1
    j = skip[:, None] + torch.arange(n, device=DEVICE)
    live = (j < ((lens + PAGE - 1) // PAGE)[:, None])[:, None, :].expand(B, H, n)
    page = table.gather(2, j.clamp(max=table.shape[2] - 1)[:, None, :].expand(B, H, n))
    seen = (j[:, :, None] * PAGE + torch.arange(PAGE, device=DEVICE)).flatten(1) < lens[:, None]
    keys, values = _pages(s, page, live)
    top, total, acc = _part(q, keys, values, seen[:, None, None, :], s["scale"])
    del keys, values
    # the prefixes, from the pages of each share's first member; every request meets every share's keys
    b = torch.arange(B, device=DEVICE)
    of = member[None, :] & (share[None, :] == torch.arange(S, device=DEVICE)[:, None])   # [S, B]
    first = torch.where(of, b, B).amin(1).clamp(max=B - 1)
    m = int(max(1, c["longest"] // PAGE))
    j = torch.arange(min(m, table.shape[2]), device=DEVICE)
    live = (j < whole[:, None]) & of.any(1)[:, None]
    page = table[first][:, :, :j.numel()]
    keys, values = _pages(s, page, live[:, None, :].expand_as(page))
    rows = q.permute(1, 0, 2, 3).reshape(1, H, B * G, D).expand(S, -1, -1, -1)
    seen = of[:, None, :, None, None] & live.repeat_interleave(PAGE, 1)[:, None, None, None, :]
    seen = seen.expand(S, 1, B, G, -1).reshape(S, 1, B * G, -1)
    top2, total2, acc2 = (x.view(S, H, B, G, -1).permute(0, 2, 1, 3, 4)
                          for x in _part(rows, keys, values, seen, s["scale"]))
    best = torch.maximum(top, top2.amax(0))
    base = torch.where(best == -math.inf, 0.0, best)
    w, w2 = torch.exp(top - base), torch.exp(top2 - base)
    total = total * w + (total2 * w2).sum(0)
    out = (acc * w + (acc2 * w2).sum(0)) / torch.where(total == 0, 1.0, total)
    return {"out": out.reshape(B, Hq, D).to(torch.bfloat16), "lse": (best + torch.log(total)).view(B, Hq)}


def _run_fork(s):
    a = s["after"]
    if own:
        import paper_2605_16839_amd as ca

        ca.sharing.fork_requests(s["cache"], s["parent"], s["seq_len"], s["page_table"], s["page_shares"],
                                 s["free_pages"], s["free_count"], (s["k_pool"], s["v_pool"]), keep_len=s["keep"],
                                 bufs=a, ws=s["ws"])
        return {**a, "k_pool": s["k_pool"], "v_pool": s["v_pool"]}
    table, shares, i32 = s["page_table"], s["page_shares"], torch.int32
    B, H, most = table.shape
    old, count = s["seq_len"].long(), s["free_count"].long()
    b = torch.arange(B, device=DEVICE)
    on = (s["parent"] >= 0) & (s["parent"] < B)
    src = torch.where(on, s["parent"].long(), 0)
    new = torch.where(on, old[src], 0)
    if s["keep"] is not None:
        new = torch.minimum(new, s["keep"].long().clamp(min=0))
    full, part = new // PAGE, new % PAGE > 0
    # who else of the parent's children holds the block that b ends in: to its end, or before b in the order
    other = on[None, :] & on[:, None] & (src[None, :] == src[:, None]) & (b[None, :] != b[:, None])
    before = (b[None, :] == src[:, None]) | ((b[None, :] < b[:, None]) & (b[:, None] != src[:, None]))
    taken = other & ((full[None, :] > full[:, None]) | ((full[None, :] == full[:, None]) & part[None, :] & before))
    h = torch.arange(H, device=DEVICE)
    last = table[src[:, None], h, full.clamp(max=most - 1)[:, None]]   # [B, H]
    held = (shares[last.clamp(min=0).long()] > 0).any(1)
    same = on & (src == b) & (new == old)
    copy = part & ~same & (taken.any(1) | held)
    need = torch.where(copy, H, 0)
    upto = need.cumsum(0)
    fits = upto <= count
    new = torch.where(copy & ~fits, full * PAGE, new)   # no page left: the whole ones are kept
    copy = copy & fits
    used = torch.where(copy, need, 0).sum()
    place = count - 1 - (upto - need)[:, None] - h
    fresh = s["free_pages"][torch.where(copy[:, None], place, 0)]
    j = torch.arange(most, device=DEVICE)
    live = (j < ((new + PAGE - 1) // PAGE)[:, None])[:, None, :].expand_as(table)
    is_copy = copy[:, None, None] & (j == full[:, None])[:, None, :]
    entry = torch.where(is_copy, fresh[:, :, None], table[src])
    a["page_table"][live] = entry[live]
    a["seq_len"].copy_(new)
    gone = (j < ((old + PAGE - 1) // PAGE)[:, None])[:, None, :] & ~same[:, None, None]
    gain = live & ~is_copy & ~same[:, None, None]
    holds = shares.long().clone()
    holds += torch.bincount(entry[gain].long(), minlength=s["pages"]) - torch.bincount(table[gone.expand_as(table)].long(), minlength=s["pages"])
    back = torch.where(holds < 0)[0]
    a["page_shares"].copy_(holds.clamp(min=0))
    left = count - used
    at = torch.arange(s["pages"], device=DEVICE)
    a["free_pages"].copy_(torch.where(at < left, s["free_pages"], a["free_pages"]))
    a["free_pages"][left + torch.arange(back.numel(), device=DEVICE)] = back.to(i32)
    a["free_count"].copy_(left + back.numel())
    to, frm = fresh[copy].flatten().long(), last[copy].flatten().long()
    for pool in (s["k_pool"], s["v_pool"]):
        pool[to] = pool[frm]
    return {**a, "k_pool": s["k_pool"], "v_pool": s["v_pool"]}


def _run_compact(s):
    a = s["after"]
    if own:
        import paper_2605_16839_amd as ca

        ca.sharing.compact_pages(s["cache"], s["seq_len"], s["page_table"], s["page_shares"], s["free_pages"],
                                 s["free_count"], (s["k_pool"], s["v_pool"]), bufs=a, ws=s["ws"])
        return {**a, "k_pool": s["k_pool"], "v_pool": s["v_pool"]}
    pages, table = s["pages"], s["page_table"]
    ids = torch.arange(pages, device=DEVICE)
    free = torch.zeros(pages, dtype=torch.bool, device=DEVICE)
    free[s["free_pages"][ids < s["free_count"]].long()] = True
    inside = pages - free.sum()   # the pages in use go below it
    frm, to = torch.where(~free & (ids >= inside))[0], torch.where(free & (ids < inside))[0]
    place = torch.where(free, -1, ids)
    place[frm] = to
    a["new_page"].copy_(place)
    live = (torch.arange(table.shape[2], device=DEVICE) < ((s["seq_len"].long() + PAGE - 1) // PAGE)[:, None])[:, None, :].expand_as(table)
    a["page_table"][live] = place[table[live].long()].to(torch.int32)
    a["page_shares"].zero_()
    a["page_shares"][place[~free]] = s["page_shares"][~free]
    a["free_count"].copy_(pages - inside)
    a["free_pages"].copy_(torch.where(ids < pages - inside, pages - 1 - ids, a["free_pages"].long()))
    for pool in (s["k_pool"], s["v_pool"]):
        pool[to] = pool[frm]
    return {**a, "k_pool": s["k_pool"], "v_pool": s["v_pool"]}


def _normed(x, weight, offset):
    y = x.float()
    y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS)
    return y * (weight.float() + (1.0 if offset else 0.0))


def _rotated(x, angle_cos, angle_sin, rotary, interleaved):
    """x [rows, heads, D], the cosines and sines [rows, 1, rotary / 2]."""
    part, rest = x[..., :rotary], x[..., rotary:]
    a, b = (part[..., 0::2], part[..., 1::2]) if interleaved else part.chunk(2, -1)
    u, w = a * angle_cos - b * angle_sin, b * angle_cos + a * angle_sin
    part = torch.stack([u, w], -1).flatten(-2) if interleaved else torch.cat([u, w], -1)
    return torch.cat([part, rest], -1)


def _run_norm(s):
    c = s["case"]
    if own:
        import paper_2605_16839_amd as ca

        q = ca.rotary_append(s["cache"], s["rotary"], s["q"], s["k"], s["v"], s["positions"], s["slot_map"],
                             (s["k_pool"], s["v_pool"]))
        return {"q": q, "k_pool": s["k_pool"], "v_pool": s["v_pool"]}
    q, k = _normed(s["q"], s["q_weight"], c["offset"]), _normed(s["k"], s["k_weight"], c["offset"])
    if c["rotary"]:   # angles in 64 bits: far positions lose their place in 32
        place = s["positions"][torch.tensor(s["pair_axis"], device=DEVICE)].t().double()
        angle = (place * s["inv_freq"].double())[:, None]
        cos, sin = angle.cos().float(), angle.sin().float()
        q, k = (_rotated(x, cos, sin, c["rotary"], c["interleaved"]) for x in (q, k))
    q, k = q.to(torch.bfloat16), k.to(torch.bfloat16)
    row, head = torch.where(s["slot_map"] >= 0)
    slot = s["slot_map"][row, head]
    s["k_pool"][slot // PAGE, slot % PAGE] = k[row, head]
    if c["layout"] == "transposed":
        s["v_pool"][slot // PAGE, :, slot % PAGE] = s["v"][row, head]
    else:
        s["v_pool"][slot // PAGE, slot % PAGE] = s["v"][row, head]
    return {"q": q, "k_pool": s["k_pool"], "v_pool": s["v_pool"]}


# ---------------------------------------------------------------------------
# the same from the definitions, in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    if case["kind"] in ("fork", "compact"):
        return None   # whole numbers, and pages that are copied bit for bit
    s = _PREPARE[case["kind"]](case, seed)
    return _exact_prefix(case, s) if case["kind"] == "prefix" else _exact_norm(case, s)


def _exact_prefix(case, s):
    """Each request by itself over all of its row: the members' rows name the shared pages too."""
    Hq, H, D = case["q_heads"], case["kv_heads"], case["dim"]
    G = Hq // H
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device=DEVICE)
    for b, n in enumerate(_prefix_plan(case)[2]):
        for kvh in range(H if n else 0):
            pages = s["page_table"][b, kvh, :_blocks(n)].long()
            k, v = s["k_pool"][pages].double(), s["v_pool"][pages].double()
            if case["layout"] == "transposed":
                v = v.transpose(1, 2)
            k, v = k.reshape(-1, D)[:n], v.reshape(-1, D)[:n]
            heads = slice(kvh * G, (kvh + 1) * G)
            x = s["q"][b, heads].double() @ k.t() * s["scale"]
            z = torch.logsumexp(x, -1)
            lse[b, heads] = z
            out[b, heads] = torch.exp(x - z[:, None]) @ v
    return {"out": out, "lse": lse}


def _exact_norm(case, s):
    R, rows, D = case["rotary"], s["q"].shape[0], case["dim"]
    turned = []
    where = s["positions"].double()
    axis = torch.tensor(s["pair_axis"], device=DEVICE, dtype=torch.long)
    for x, w in ((s["q"], s["q_weight"]), (s["k"], s["k_weight"])):
        x = x.double()
        x = x / (x.pow(2).sum(-1, keepdim=True) / D + EPS).sqrt() * (w.double() + (1 if case["offset"] else 0))
        y = x.clone()
        for i in range(R // 2):   # pair i turns by its axis' place times its frequency
            angle = where[axis[i]] * s["inv_freq"][i].double()
            at = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + R // 2)
            turn = torch.polar(torch.ones_like(angle), angle).view(rows, 1)
            z = torch.complex(x[..., at[0]], x[..., at[1]]) * turn
            y[..., at[0]], y[..., at[1]] = z.real, z.imag
        turned.append(y)
    pool = s["k_pool"].double().view(-1, D)
    for h in range(case["kv_heads"]):
        kept = s["slot_map"][:, h] >= 0
        pool[s["slot_map"][kept, h]] = turned[1][kept, h]
    return {"q": turned[0], "k_pool": pool.view(s["k_pool"].shape), "v_pool": None}
