"""Row counts that are upper bounds: n_rows only has to reach rows[batch], and a captured call keeps it at its capacity."""
import numpy as np
import pytest
import torch

import paged_ref as ref
from test_paged_gpu import DEV, Setup

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2609_03430_gb300 as ra


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("n_rows", [1000, 2 ** 27, 2 ** 27 - 32])
def test_rows_far_below_their_upper_bound(fp8, n_rows):
    """8.4 million CTAs of 256 threads (2^31 threads and more), of which a handful have rows: those go where they belong, nothing else moves."""
    lens, KVH, D = [70, 0, 33], 8, 64
    s = Setup(lens, KVH=KVH, G=1, D=D, page=16, fp8=fp8)
    k, v = torch.cat(s.k[0]).to(DEV), torch.cat(s.v[0]).to(DEV)
    rows = torch.tensor([0, 70, 70, 103], dtype=torch.int32, device=DEV)
    ra.ra_paged_write(s.ctx, 0, k.data_ptr(), v.data_ptr(), KVH * D, D, 3, rows.data_ptr(), n_rows, *s._seqs())
    back = torch.full((2, 110, KVH, D), 7.0, dtype=torch.bfloat16, device=DEV)
    ra.ra_paged_read(s.ctx, 0, back[0].data_ptr(), back[1].data_ptr(), KVH * D, D, 3, rows.data_ptr(), n_rows, *s._seqs())
    assert np.array_equal(ref.wide(back[0, :103]), ref.held(ref.wide(k), fp8))
    assert np.array_equal(ref.wide(back[1, :103]), ref.held(ref.wide(v), fp8))
    assert (back[:, 103:] == 7).all()
    s.done()


def test_rows_read_back_over_each_other_are_refused():
    """Both strides a row's length: every head's row 1 would lie on the next head's row 0."""
    s = Setup([40, 7], KVH=4, G=1, D=64, page=16)
    s.write()
    out = torch.zeros(2, 47 * 64 * 4, dtype=torch.bfloat16, device=DEV)
    rows = torch.tensor([0, 40, 47], dtype=torch.int32, device=DEV)
    for row, head in ((64, 64), (128, 64), (192, 64), (64, 128), (64, 46 * 64)):
        with pytest.raises(ra.RAError) as e:
            ra.ra_paged_read(s.ctx, 0, out[0].data_ptr(), out[1].data_ptr(), row, head, 2, rows.data_ptr(), 47, *s._seqs())
        assert e.value.code == ra.RA_ERR_INVALID_ARG
    torch.cuda.synchronize()
    assert (out == 0).all()
    for row, head in ((256, 64), (64, 47 * 64)):
        ra.ra_paged_read(s.ctx, 0, out[0].data_ptr(), out[1].data_ptr(), row, head, 2, rows.data_ptr(), 47, *s._seqs())
        k = out[0].view(47, 4, 64) if head == 64 else out[0].view(4, 47, 64).transpose(0, 1)
        assert np.array_equal(ref.wide(k), ref.held(ref.wide(torch.cat(s.k[0])), True))
    s.done()
