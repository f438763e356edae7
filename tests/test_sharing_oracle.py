"""The oracle of requests that share pages, pinned by hand-worked steps and invariants (CPU)."""
import numpy as np
import pytest

from oracle import serving, sharing


def test_a_prompt_becomes_three_requests():
    table = np.full((3, 1, 3), -1)
    table[0, 0, :2] = 4, 7                     # 100 tokens: page 4 is full, 36 in page 7
    s = sharing.fork_requests([0, 0, 0], None, [100, 0, 0], table, np.zeros(9), [1, 2, 3, 5], 9)
    assert s["seq_len"].tolist() == [100, 100, 100]
    assert s["page_table"][:, 0, :2].tolist() == [[4, 7], [4, 5], [4, 3]]
    assert s["copies"] == [(7, 5), (7, 3)] and s["free"] == [1, 2]
    assert s["page_shares"].tolist() == [0, 0, 0, 0, 2, 0, 0, 0, 0]


def test_beams_swap_and_end():
    table = np.array([[[0, 1]], [[0, 2]], [[0, 3]]])      # one prompt page, a tail each
    shares = [2, 0, 0, 0, 0]
    # request 0 goes on from 1, 1 from 1, 2 ends; so 1's tail is copied for 0, and 0's and 2's are free
    s = sharing.fork_requests([1, 1, -1], None, [70, 80, 90], table, shares, [4], 5)
    assert s["seq_len"].tolist() == [80, 80, 0]
    assert s["page_table"][:2, 0].tolist() == [[0, 4], [0, 2]] and s["copies"] == [(2, 4)]
    assert s["page_shares"].tolist() == [1, 0, 0, 0, 0] and s["free"] == [1, 3]
    # two rows change places: nothing is copied
    s = sharing.fork_requests([1, 0, 2], None, [70, 80, 90], table, shares, [], 5)
    assert s["page_table"][:2, 0].tolist() == [[0, 2], [0, 1]] and not s["copies"]
    assert s["page_shares"].tolist() == shares and s["free"] == []


def test_no_page_left_keeps_the_whole_ones():
    table = np.array([[[0, 1]], [[-1, -1]], [[-1, -1]]])
    s = sharing.fork_requests([0, 0, 0], None, [70, 0, 0], table, [0, 0, 0], [2], 3)
    assert s["seq_len"].tolist() == [70, 70, 64] and s["free"] == []
    assert s["page_shares"].tolist() == [2, 0, 0]


def test_shorter_forks():
    table = np.array([[[0, 1]], [[-1, -1]], [[-1, -1]]])
    # 30 of 70 tokens: page 0 is still 0's to the end, so it is copied; 64: shared
    s = sharing.fork_requests([0, 0, 0], [70, 30, 64], [70, 0, 0], table, [0] * 4, [2, 3], 4)
    assert s["seq_len"].tolist() == [70, 30, 64] and s["copies"] == [(0, 3)]
    assert s["page_shares"].tolist() == [1, 0, 0, 0]
    # 0 itself goes back to 30 tokens, alone: in place, and page 1 is free
    s = sharing.fork_requests([0, -1, -1], [30, 0, 0], [70, 0, 0], table, [0] * 4, [2, 3], 4)
    assert s["seq_len"].tolist() == [30, 0, 0] and not s["copies"] and s["free"] == [2, 3, 1]


@pytest.mark.parametrize("seed", range(20))
def test_holds_are_conserved(seed):
    """Over steps: a page's holders are counted by the tables, and no page is lost or given twice."""
    rng = np.random.default_rng(seed)
    B, H, most, pages = 6, 2, 5, 80
    table, lens = np.full((B, H, most), -1), np.zeros(B, dtype=np.int64)
    shares, free = np.zeros(pages, dtype=np.int64), list(rng.permutation(pages))
    for _ in range(12):
        new = rng.integers(0, 70, B)
        a = serving.assign_slots(new, int(new.sum()), lens, table, free, pages)
        lens, table, free = a["seq_len"], a["page_table"], a["free"]
        parent, keep = rng.integers(-1, B, B), rng.integers(0, 330, B) if rng.random() < 0.5 else None
        s = sharing.fork_requests(parent, keep, lens, table, shares, free, pages)
        lens, table, shares, free = s["seq_len"], s["page_table"], s["page_shares"], s["free"]
        holds = np.zeros(pages, dtype=np.int64)
        last = []
        for b in range(B):
            for j in range(-(-lens[b] // 64)):
                for h in range(H):
                    holds[table[b, h, j]] += 1
                    if lens[b] - 64 * j < 64:
                        last.append(table[b, h, j])
        assert np.array_equal(np.maximum(holds - 1, 0), shares)
        assert sorted(free) == np.flatnonzero(holds == 0).tolist()
        assert (holds[last] == 1).all()        # whoever appends writes to a page of its own
        c = sharing.compact_pages(lens, table, shares, free, pages)
        assert sorted(c["new_page"][holds > 0]) == list(range(int((holds > 0).sum())))
        table, shares, free = c["page_table"], c["page_shares"], c["free"]


def test_compaction_by_hand():
    table = np.array([[[5, 2, 9]]])
    s = sharing.compact_pages([130], table, [0, 0, 1, 0, 0, 3, 0], [0, 3, 6, 6, -1, 99], 7)
    # in use: 1, 2, 4, 5: the ids below 4 are 0..3, so 4 goes to 0 and 5 to 3
    assert s["new_page"].tolist() == [-1, 1, 2, -1, 0, 3, -1]
    assert s["page_table"][0, 0].tolist() == [3, 2, 9] and s["free"] == [6, 5, 4]
    assert s["page_shares"].tolist() == [0, 0, 1, 3, 0, 0, 0]


def test_norm_by_hand():
    assert np.allclose(sharing.normed(np.array([3.0, 4.0]), np.array([1.0, 2.0]), 0.0),
                       np.array([3, 8]) / np.sqrt(12.5))


def test_prefix_rows():
    table = np.arange(12).reshape(4, 1, 3)
    rows = sharing.prefix_rows(table, [130, 128, 64, 200], [0, 0, 0, 1], [129, 500])
    assert rows[:, 0].tolist() == [[0, 1, 2], [0, 1, 5], [6, 7, 8], [9, 10, 11]]
