"""A sequence whose length is taken back and whose positions are written again: rows and attention are the new ones alone; a
page's bounds are those of every key written there since its first position was."""
import numpy as np
import pytest
import torch

import paged_ref as ref
from test_paged_gpu import Setup

pytestmark = pytest.mark.gpu


def chosen(q, pages, top):
    """Page indices by the definition, the rows of each page given apart."""
    unit_q = 2.0 ** ref.power_of_two_scale(np.abs(q).max(), 127.0, -120)
    qi = np.rint(q / unit_q)
    score = []
    for rows in pages:
        if not np.isfinite(rows).all():
            score.append((1, 0.0))
            continue
        lo, hi = rows.min(0), rows.max(0)
        unit = 2.0 ** ref.power_of_two_scale(max(np.abs(lo).max(), np.abs(hi).max()), 127.0, -120)
        whole = int(np.where(qi > 0, qi * np.ceil(hi / unit), qi * np.floor(lo / unit)).sum())
        score.append((0, float(np.float32(whole)) * unit))
    return sorted(sorted(range(len(pages)), key=lambda i: (-score[i][0], -score[i][1], i))[:top])


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("left", [5, 0.25, float("nan")])
def test_length_taken_back(fp8, left):
    """Page 2 of 6 is filled, then taken back to its fifth row and written again: by usual keys after keys `left` times their size, or
    after one that was not finite."""
    P, n, D = 16, 96, 64
    s = Setup([n], KVH=2, G=2, D=D, page=P, fp8=fp8, bounds=True)
    new = s.k[0][0].clone()
    dropped = new.clone()
    dropped[37:48] *= 1.0 if left != left else left
    if left != left:
        dropped[40, :, 7] = left
    s.k[0][0] = dropped
    s.write([48], [48])                      # three pages
    s.k[0][0] = new
    s.write([3], [40])                       # back to 37, on to 40
    s.write([1], [41])
    s.write([n - 41], [n])
    k, _ = s.read()
    assert np.array_equal(k, ref.held(ref.wide(new), fp8))
    s.check_attention(*s.dense())
    pages = [[ref.wide(new[i:i + P, h]) for i in range(0, n, P)] for h in range(2)]
    since = [[np.concatenate([p, ref.wide(dropped[37:48, h])]) if i == 2 else p for i, p in enumerate(pages[h])] for h in range(2)]
    for top in range(1, 6):
        sel = s.select(top, 0, 0)[0].tolist()
        assert sel == [chosen(ref.wide(s.q)[0, 2 * h:2 * h + 2], since[h], top) for h in range(2)], top
        if left != left:
            assert all(2 in x for x in sel)
    s.write([n - 32], [n])                   # the page from its first position: what it holds, no more
    for top in range(1, 6):
        sel = s.select(top, 0, 0)[0].tolist()
        assert sel == [chosen(ref.wide(s.q)[0, 2 * h:2 * h + 2], pages[h], top) for h in range(2)], top
        assert sel == [ref.choose(ref.wide(s.q)[0, 2 * h:2 * h + 2], ref.wide(new[:, h]), P, top, 0, 0) for h in range(2)]
    s.done()


def test_a_shorter_length_without_a_write():
    """Lengths alone set back: the last page's bounds are of more keys than count, its rows are not read."""
    s = Setup([96], KVH=1, G=2, D=64, page=16, bounds=True)
    s.write()
    s.lens = [70]
    s.dlens[0] = 70
    full = s.k[0][0]
    pages = [ref.wide(full[i:i + 16, 0]) for i in range(0, 80, 16)]
    for top in range(1, 5):
        assert s.select(top, 0, 0)[0, 0].tolist() == chosen(ref.wide(s.q)[0], pages, top)
    s.k[0][0] = full[:70]
    s.check_attention(*s.dense())
    s.done()
