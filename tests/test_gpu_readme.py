"""The README's code of the serving step, run as it stands: samples of one prompt, forked a token before a page
is full, so that each request's first token of its own is in that page."""
import os
import re

import pytest
import torch

pytestmark = pytest.mark.gpu

ca = pytest.importorskip("paper_2605_16839_amd")
README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")
BF16_HALF = 2.0 ** -8


def test_samples_of_one_prompt(monkeypatch):
    with open(README) as f:
        blocks = re.findall(r"```python\n(.*?)```", f.read(), re.S)
    names = {}
    serving = next(i for i, b in enumerate(blocks) if "assign_slots" in b)
    for b in blocks[:serving + 1]:
        exec(b, names)
    step = blocks[serving][blocks[serving].index("new_len ="):]
    while int(names["state"]["seq_len"][0]) < 63:
        exec(step, names)
    seen = []

    def call(cache, q, pools, page_table, kv_len, share, share_len, scale, **kw):
        out, lse = prefix(cache, q, pools, page_table, kv_len, share, share_len, scale, **kw)
        seen.append((out, ca.decode_attention(cache, q, pools, page_table, kv_len, scale)[0], kv_len.tolist(), share_len.tolist()))
        return out, lse

    prefix = ca.sharing.prefix_decode_attention
    monkeypatch.setattr(ca.sharing, "prefix_decode_attention", call)
    for b in blocks[serving + 1:]:
        exec(b, names)
    torch.cuda.synchronize()
    assert len(seen) == 1
    out, want, lens, share_len = seen[0]
    assert lens == [64] * 64 and share_len == [63]      # a token of each request's own, behind what it shares
    # both are within a bf16 half step and a little of the exact result
    assert ((out.float() - want.float()).abs() <= 2.1 * BF16_HALF * want.float().abs() + 2.0 ** -14).all()
    assert not torch.equal(out[0], out[1])              # q differs, and so does the last key
