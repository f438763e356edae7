"""The serving step around the paged cache (float64 and plain Python), test infrastructure only.

* ``assign_slots`` / ``release_pages`` replay the step request by request on a
  list used as a stack: a page is popped whenever a block opens for a head.
  Parity: pinned by hand-worked steps and by conservation of the pages
  (tests/test_serving_oracle.py).
* ``rotate`` turns pairs as complex numbers in float64.  Parity: pinned by the
  angle-difference property of rotary positions (q.k depends on the distance).
* ``decode_attention`` is the softmax of one query per head over explicitly
  gathered keys.  Parity: pinned by ``oracle.chunk_attention`` with a chunk of one token.
"""
from __future__ import annotations

from typing import List, Optional, Sequence

import numpy as np

from .bf16 import bf16_to_f64

PAGE = 64


def release_pages(release, seq_len, page_table, free: Sequence[int], capacity: int,
                  max_blocks: int):
    """(seq_len, free list) after the requests with release != 0 ended."""
    Hkv = page_table.shape[1]
    free, out, wanted = list(free), [int(x) for x in seq_len], len(free)
    for b, flag in enumerate(release):
        n = int(seq_len[b])
        if not flag or n < 0 or n > PAGE * max_blocks:
            continue
        blocks = -(-n // PAGE)
        wanted += blocks * Hkv
        if blocks and wanted > capacity:
            continue
        free += [int(page_table[b, h, j]) for j in range(blocks) for h in range(Hkv)]
        out[b] = 0
    return out, free


def assign_slots(new_len, num_tokens: int, seq_len, page_table, free: Sequence[int],
                 num_pages: int) -> dict:
    """The step's tables; ``free`` is a list whose last element is taken first."""
    B, Hkv, max_blocks = page_table.shape
    table = np.array(page_table, dtype=np.int64)
    free = list(free)
    slot = np.full((num_tokens, Hkv), -1, dtype=np.int64)
    pos = np.zeros(num_tokens, dtype=np.int64)
    indptr, granted, lens = [0], [], []
    row, wanted, there = 0, 0, len(free)
    for b in range(B):
        old, add = int(seq_len[b]), int(new_len[b])
        first = row
        row += max(add, 0)
        indptr.append(min(row, num_tokens))
        ok = old >= 0 and add >= 0 and old + add <= PAGE * max_blocks and row <= num_tokens
        if ok:
            need = (-(-(old + add) // PAGE) - -(-old // PAGE)) * Hkv
            wanted += need
            ok = need == 0 or wanted <= there
        granted.append(add if ok else 0)
        lens.append(old + (add if ok else 0))
        if not ok:
            continue
        for i in range(add):
            p = old + i
            if p % PAGE == 0:
                for h in range(Hkv):
                    table[b, h, p // PAGE] = free.pop()
            pos[first + i] = p
            for h in range(Hkv):
                page = table[b, h, p // PAGE]
                if 0 <= page < num_pages:
                    slot[first + i, h] = page * PAGE + p % PAGE
    return dict(slot_map=slot, positions=pos, token_indptr=np.array(indptr), granted=np.array(granted),
                seq_len=np.array(lens), free_count=np.array([len(free)]), page_table=table, free=free)


def rotate(x: np.ndarray, positions: np.ndarray, inv_freq: np.ndarray,
           pair_axis: Optional[Sequence[int]] = None, interleaved: bool = False) -> np.ndarray:
    """x [T, H, D] float64; positions [axes, T]; inv_freq [pairs] (as float32 values)."""
    y = np.array(x, dtype=np.float64)
    n = len(inv_freq)
    for i in range(n):
        axis = 0 if pair_axis is None else pair_axis[i]
        turn = np.exp(1j * positions[axis].astype(np.float64) * float(inv_freq[i]))[:, None]
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
        z = (x[..., a] + 1j * x[..., b]) * turn
        y[..., a], y[..., b] = z.real, z.imag
    return y


def decode_attention(q_bits, k_pool_bits, v_pool_bits, page_table, kv_len, sm_scale: float,
                     tables: Optional[List[List[List[int]]]] = None, group_size: int = 0):
    """out [B, Hq, D], lse [B, Hq], and what bounds a kernel's rounding: sum_j w_j |v_j|
    [B, Hq, D] (w the softmax weights) and max_j sm_scale * sum_d |q_d k_jd| [B, Hq].
    v_pool is token-major here.  ``tables[b][g]`` lists blocks; None: all."""
    q = bf16_to_f64(q_bits)
    B, Hq, D = q.shape
    Hkv = page_table.shape[1]
    gs = group_size or Hq // Hkv
    out, mass = np.zeros(q.shape), np.zeros(q.shape)
    lse, size = np.full((B, Hq), -np.inf), np.zeros((B, Hq))
    for b in range(B):
        n = int(kv_len[b])
        for g in range(Hq // gs):
            kvh = g * gs // (Hq // Hkv)
            blocks = list(range(-(-n // PAGE))) if tables is None else tables[b][g]
            keys = [(page_table[b, kvh, j], min(PAGE, n - PAGE * j)) for j in blocks]
            keys = [(p, r) for p, r in keys if r > 0]
            if not keys:
                continue
            k = np.concatenate([bf16_to_f64(k_pool_bits[p, :r]) for p, r in keys])
            v = np.concatenate([bf16_to_f64(v_pool_bits[p, :r]) for p, r in keys])
            for h in range(g * gs, (g + 1) * gs):
                x = sm_scale * (k @ q[b, h])
                m = x.max()
                w = np.exp(x - m)
                lse[b, h] = m + np.log(w.sum())
                out[b, h] = w @ v / w.sum()
                mass[b, h] = w @ np.abs(v) / w.sum()
                size[b, h] = sm_scale * (np.abs(k) @ np.abs(q[b, h])).max()
    return out, lse, mass, size
