"""Long launches in which no tile may be lost: with queries of zero every row has the same weight, so that the log sum is log n
and an output counts the tiles whose values it has.  Checked for every sequence and head, across the borders of shares and the
joins; the tolerances are those of the last steps alone, and a single row that is missing (or counted twice) is outside them."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2609_03430_gb300 as ra

DEV = "cuda"

CASES = [
    (True, 64, 64, 8, 2, [40000, 7, 0, 31111, 100] * 8 + [99999]), (True, 128, 16, 8, 4, [40000, 7, 0, 31111, 100] * 4),
    (True, 128, 64, 8, 8, [131071]), (True, 64, 16, 1, 1, [131071, 64]), (True, 128, 128, 2, 12, [60001] * 10),
    (False, 64, 64, 8, 4, [20000, 64, 15001] * 10), (False, 64, 128, 8, 16, [70000] * 5), (False, 128, 64, 8, 8, [131071]),
    (False, 128, 16, 4, 5, [38912, 1, 20003] * 6), (False, 128, 32, 8, 4, [1 + 97 * b for b in range(200)]),
    (True, 64, 32, 8, 4, [1 + 97 * b for b in range(200)]),
]


@pytest.mark.parametrize("fp8, D, page, KVH, G, lens", CASES, ids=[str(i) for i in range(len(CASES))])
def test_every_tile_counts_once(fp8, D, page, KVH, G, lens):
    B, n = len(lens), sum(lens)
    counts = [-(-x // page) for x in lens]
    cache = ra.PagedCache(1, KVH * G, KVH, D, page, sum(counts), B, max(lens), int(fp8))
    gen = torch.Generator().manual_seed(n)
    order = torch.randperm(sum(counts), generator=gen, dtype=torch.int32)
    table = torch.zeros(B, max(counts), dtype=torch.int32)
    for b, at in enumerate(np.cumsum([0] + counts[:-1])):
        table[b, :counts[b]] = order[at:at + counts[b]]
    table, dl = table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV)
    rows = torch.tensor(np.cumsum([0] + lens), dtype=torch.int32, device=DEV)
    k = torch.randn(n, KVH, D, device=DEV).bfloat16()
    # row i of head h: 1 in channel (i // 16 + 5 h) % D, 0 elsewhere (16 rows divide every tile)
    i = torch.cat([torch.arange(x) for x in lens]).to(DEV)
    channel = (i[:, None] // 16 + 5 * torch.arange(KVH, device=DEV)) % D
    v = torch.zeros(n, KVH, D, dtype=torch.bfloat16, device=DEV).scatter_(2, channel[..., None], 1.0)
    seqs = (dl.data_ptr(), table.data_ptr(), table.shape[1])
    ra.ra_paged_write(cache.ctx, 0, k.data_ptr(), v.data_ptr(), KVH * D, D, B, rows.data_ptr(), n, *seqs)
    q = torch.zeros(B, KVH * G, D, dtype=torch.bfloat16, device=DEV)
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device=DEV)
    ra.ra_paged_attn(cache.ctx, 0, q.data_ptr(), KVH * G * D, D, out.data_ptr(), lse.data_ptr(), B, *seqs)
    ra.ra_paged_check(cache.ctx)
    out, lse = out.double().cpu().numpy().reshape(B, KVH, G, D), lse.double().cpu().numpy().reshape(B, KVH, G)
    for b, x in enumerate(lens):
        if x == 0:
            assert (out[b] == 0).all() and np.isneginf(lse[b]).all()
            continue
        # the weights' sum is exact (n terms of 2^-8, with the reference 8 above); log2f (1 unit in the last place), its sum with
        # the reference (half a unit), the product with log 2 and that constant (2^-24 and 2^-25 of the result)
        bits = math.log2(x)
        tol = math.log(2) * float(np.spacing(np.float32(abs(bits - 8))) + np.spacing(np.float32(bits)) / 2) + 1.5 * 2.0 ** -24 * math.log(x)
        assert math.log(x + 1) - math.log(x) > 2 * tol
        assert (np.abs(lse[b] - math.log(x)) <= tol).all(), (b, x, np.abs(lse[b] - math.log(x)).max(), tol)
        sets = np.bincount(np.arange(x) // 16 % D, minlength=D)
        for h in range(KVH):
            # one of the roundings to bf16 of what sums and divisions in 32 bits may give (2^-20)
            want = torch.from_numpy(np.roll(sets, 5 * h) / x)
            lo, hi = ((want * (1 + e)).float().bfloat16().double().numpy() for e in (-2.0 ** -20, 2.0 ** -20))
            assert ((out[b, h] == lo) | (out[b, h] == hi)).all(), (b, h)
        most = sets.max() / 16  # 16 rows more or less of a channel are 1 / most of it: a step of bf16 or more
        assert 1 / most >= 2.0 ** -7
    cache.close()
