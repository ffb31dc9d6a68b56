"""Attention over V rows near bf16's largest values, among rows of usual size: products of weights and values stay within 32
bits where the outputs do, and the other rows still count in the sum of the softmax, within a warp and where parts are
joined."""
import numpy as np
import pytest
import torch

from test_paged_gpu import Setup

pytestmark = pytest.mark.gpu

SHAPES = pytest.mark.parametrize("lens, KVH", [([3000], 1), ([1500] * 16, 8), ([40, 100], 2)],
                                 ids=["joined", "several tiles a warp", "short"])


def one_large_row(fp8, at, lens, KVH, others=1.0):
    """The large row's logit is 12, the rest's about N(0, 1): 1500 of them hold 1.5% of the weight, 3000 hold 3%."""
    s = Setup(lens, KVH=KVH, G=2, D=64, page=32, fp8=fp8)
    large = [(x.double().clamp(-3, 3) * 2.0 ** 125).bfloat16() for x in s.v[0]]
    s.v = [[(x.double() * others).bfloat16() for x in s.v[0]]]
    for b, n in enumerate(lens):
        i = min(at, n // 2)
        for h in range(KVH):
            q = s.q[b, 2 * h].double()
            s.k[0][b][i, h] = (q * 12.0 * 8.0 / (q @ q)).bfloat16()
        s.v[0][b][i] = large[b][i]
    s.write()
    out, lse = s.dense()
    assert bool(torch.isfinite(out.float()).all()) and np.isfinite(lse.cpu().numpy()).all()
    s.check_attention(out, lse)
    s.done()


@SHAPES
@pytest.mark.parametrize("at", [5, 700, -3])
def test_one_row_of_the_largest_values_in_bf16(at, lens, KVH):
    """A weight may not pass 1: 2^7 times a row of 2^126 is infinite, whatever the sum it is divided by."""
    one_large_row(False, at, lens, KVH)


@SHAPES
@pytest.mark.parametrize("at", [5, 700, -3])
@pytest.mark.parametrize("others", [1.0, 0.0, 2.0 ** -100, 2.0 ** 60])
def test_one_row_of_the_largest_values_in_8_bits(at, lens, KVH, others):
    """The unit of the value sums follows logit + log2 of the V row's scale, 2^119 here and 2^-60 at least: the other rows may
    lie up to 2^-180 below it and still count in the softmax's sum."""
    one_large_row(True, at, lens, KVH, others)


def test_rows_of_the_largest_values_alone():
    """All rows large, in 8 bits: the outputs are, too, and stay finite."""
    s = Setup([900, 33], KVH=2, G=3, D=64, page=16, fp8=True)
    s.v = [[(x.double().clamp(-3, 3) * 2.0 ** 125).bfloat16() for x in s.v[0]]]
    s.write()
    out, lse = s.dense()
    assert bool(torch.isfinite(out.float()).all()) and np.isfinite(lse.cpu().numpy()).all()
    s.check_attention(out, lse)
    s.done()
