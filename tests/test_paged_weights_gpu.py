"""How many bits the weights of the softmax keep: values that nearly cancel leave their rounding bare, where values of one
sign hide it below the output's."""
import numpy as np
import pytest
import torch

import paged_ref as ref
from test_paged_gpu import Setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("KVH, G", [(2, 1), (1, 11)])
def test_pairs_of_opposite_values(fp8, D, KVH, G):
    """Rows in pairs of logits a and b and of values 1 and -1: the output is tanh((a - b) / 2), 2^-9 or 2^-8 here.

    One product per logit, exact in both formats (values of 4 significant bits), so an output is off by: its rounding to bf16 (2^-9
    of it, doubled); the weights' parts (2^-16 in bf16, whose second part has 8 bits; 2^-22 in 8 bits), the logit's products by scale and by log2
    e and the difference to the reference (4 * 2^-24), 2^x (2^-22), and sums in 32 bits whose terms are all of a size (2^-20 of them)."""
    lens = [2, 34, 700, 4096, 30000] * 3
    s = Setup(lens, KVH=KVH, G=G, D=D, page=64, fp8=fp8)
    rng = np.random.default_rng(D)
    for b, n in enumerate(lens):
        eighths = rng.integers(8, 14, size=(KVH, 1))
        pair = np.concatenate([eighths, eighths + 1], 1) / 8.0 * 2.0 ** -5  # logits 1/32 to 1.75/32, 1/256 apart
        k = torch.zeros(n, KVH, D)
        k[:, :, 3] = torch.from_numpy(np.tile(pair.T, (n // 2, 1)))
        s.k[0][b] = k.bfloat16()
        s.v[0][b] = torch.tensor([1.0, -1.0]).repeat(n // 2)[:, None, None].expand(n, KVH, D).bfloat16().contiguous()
    s.q[:] = 0
    s.q[:, :, 3] = 1.0
    s.q[:, G // 2::G, 3] = 2.0  # (a head of its own weights in each group)
    s.write()
    out, lse = s.dense(scale=1.0)
    out = ref.wide(out)
    for b in range(len(lens)):
        for h in range(KVH * G):
            logit = ref.wide(s.q[b, h, 3]) * ref.wide(s.k[0][b][:2, h // G, 3])
            want = np.tanh((logit[0] - logit[1]) / 2)
            assert 2.0 ** -10 < abs(want) < 2.0 ** -6
            tol = 2.0 ** -8 * abs(want) + (2.0 ** -22 if fp8 else 2.0 ** -16) + 4 * 2.0 ** -24 + 2.0 ** -22 + 2.0 ** -20
            assert (np.abs(out[b, h] - want) <= tol).all(), (b, h, want, out[b, h, 0], tol)
    s.done()
