"""Shapes that take a path of their own: bounds kept by a write of so many pages that each head has one warp, the tiles of more
than 32 sequences of 128 channels (and 128 threads in bf16), and the timed cases against their definitions in 64 bits."""
import importlib.util
import os
import random

import numpy as np
import pytest
import torch

import paged_ref as ref
from test_paged_gpu import Setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("D, page, lens", [(64, 16, [20011, 0, 777]), (128, 32, [25000, 17003])])
def test_bounds_of_many_pages_written_at_once(fp8, D, page, lens):
    """1300 pages and more of 8 heads in one call (from 9728 page heads on, a warp per head), and a second call that continues pages."""
    s = Setup(lens, KVH=8, G=2, D=D, page=page, fp8=fp8, bounds=True)
    assert sum(n // page for n in lens) * 8 >= 64 * 152
    first = [n - n // 50 for n in lens]
    s.write(first, first)
    s.write([n - f for n, f in zip(lens, first)])
    k, v = s.read()
    assert np.array_equal(k, ref.held(ref.wide(torch.cat(s.k[0])), fp8))
    for top in (1, 40, 333):
        sel = s.select(top, 1 if top > 1 else 0, 0).cpu().numpy()
        for b, n in enumerate(lens):
            for h in (0, 3, 7):
                want = ref.choose(ref.wide(s.q)[b, 2 * h:2 * h + 2], ref.wide(s.k[0][b][:, h]), page, top, 1 if top > 1 else 0, 0) if n else []
                assert sel[b, h].tolist() == want + [-1] * (top - len(want)), (b, h, top)
    s.done()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("B", [32, 33, 129, 512])
def test_dense_of_many_sequences_of_128_channels(fp8, B):
    lens = [(53 * b) % 211 for b in range(B)]
    s = Setup(lens, KVH=2, G=3, D=128, page=32, fp8=fp8)
    s.write()
    s.check_attention(*s.dense())
    s.done()


def cases():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "perf", "operators.py")
    spec = importlib.util.spec_from_file_location("paged_operator_cases", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


NAMES = ["write one token bf16", "write batch 64 fp8", "dense one user bf16", "dense batch 16 fp8", "sparse one user fp8", "sparse batch 16 bf16"]


@pytest.mark.parametrize("which", NAMES + list(range(8)))
def test_timed_cases_are_their_definitions(which):
    """Listed cases of up to 0.2 GB, and drawn ones: held rows and chosen pages are equal; outputs are off by their rounding to bf16
    (2^-9, doubled, as an error before it can move it) and by logits summed in 32 bits, D * 2^-24 of sum |q k| scale, at most 40 for these inputs
    (twice on a weight, of values that average 1.1 at most), log sums by the logits' part and 2^-19."""
    m = cases()
    m.own = True
    if isinstance(which, str):
        case = next(c for c in m.listed() if c["name"] == which)
    else:
        rng = random.Random(which)
        case = m.draw(rng)
        while m.work(case)["bytes"] > 0.1e9:
            case = m.draw(rng)
    want = m.exact(case, 11)
    if want is None:
        pytest.skip("too large for the definition")
    state = m.prepare(case, 11)
    got = m.run(state)
    state["ra"].ra_paged_check(state["ctx"])
    if case["op"] == "write":
        assert all(torch.equal(g.double(), w) for g, w in zip(got, want))
        return
    if case["op"] == "sparse":
        assert torch.equal(got[0], want[0])
        got, want = got[1:], want[1:]
    out, lse = got[0].double(), got[1].double()
    logits = case["head_dim"] * 2.0 ** -24 * 40
    err = (out - want[0]).abs()
    assert bool((err <= 2.0 ** -8 * want[0].abs() + 2.2 * logits).all()), err.max()
    assert float(err.norm() / want[0].norm()) < 2.0 ** -9 + 2.0 ** -12
    empty = torch.isneginf(want[1])
    assert torch.equal(empty, torch.isneginf(lse))
    assert bool(((lse - want[1])[~empty].abs() <= logits + 2.0 ** -19 * want[1][~empty].abs().clamp_min(1)).all())
