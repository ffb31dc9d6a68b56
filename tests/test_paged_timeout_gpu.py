"""A bounded wait of the paged attention that runs out: the call's check reports it once, the heads whose rows did not arrive
read NaN (not what an earlier call left), the others are right, and the next call is right everywhere.

The wait runs out safely: one share of a probe launch expects 16 bytes more of a tile than it copies, all its copies are
ordinary ones within the pool, and its waits are bounded at 1 ms."""
import pytest
import torch

from test_paged_gpu import DEV, Setup

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2609_03430_gb300 as ra


def shares_of(lens, KVH, tile):
    """Per (sequence, KV head): its first tile and tiles, tiles laid end to end; and the shares' begins."""
    warps = 8 * torch.cuda.get_device_properties(0).multi_processor_count
    heads, at = {}, 0
    for b, n in enumerate(lens):
        for h in range(KVH):
            heads[b, h] = (at, -(-n // tile))
            at += -(-n // tile)
    W = min(warps, at)
    return heads, [w * (at // W) + min(w, at % W) for w in range(W + 1)]


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("lens", [[20011], [700, 0, 33, 5000] * 20, [1 + b % 64 for b in range(512)]], ids=["one", "ragged", "many short"])
def test_a_wait_that_runs_out(fp8, lens):
    KVH, G, D = 8 if len(lens) > 1 else 2, 2, 64
    s = Setup(lens, KVH=KVH, G=G, D=D, page=16, fp8=fp8)
    s.write()
    out, lse = s.dense()
    other = s.q.flip(0) if len(lens) > 1 else -s.q
    s.dense(q=other)  # (what records and buffers hold next is not this call's)
    q = s.q.to(DEV)
    heads, begin = shares_of(lens, KVH, 64 if fp8 else 32)
    for share, tile in ((0, 0), (len(begin) // 2, 0), (len(begin) // 2 + 1, 1), (len(begin) - 2, 0)):
        first = begin[share] + tile
        tile = tile if first < begin[share + 1] else 10 ** 6  # (a share of one tile: nothing runs out)
        o, l = s.outputs()
        ra.ra_paged_debug_timeout_probe(s.ctx, 0, q.data_ptr(), KVH * G * D, D, o.data_ptr(), l.data_ptr(), s.B, *s._seqs(), share, tile, 1_000_000)
        if tile < 10 ** 6:
            with pytest.raises(ra.RAError) as e:
                ra.ra_paged_check(s.ctx)
            assert e.value.code == ra.RA_ERR_DEVICE_TIMEOUT and "bounded wait" in str(e.value)
        ra.ra_paged_check(s.ctx)  # reported once
        gone = torch.zeros(s.B, KVH, dtype=torch.bool)
        for (b, h), (at, n) in heads.items():
            # the tile, what follows it in the share, and what came before it of the same head
            gone[b, h] = tile < 10 ** 6 and at + n > first and at < begin[share + 1]
        gone = gone.repeat_interleave(G, 1).to(DEV)
        assert torch.isnan(o[gone]).all() and torch.isnan(l[gone]).all()
        assert torch.equal(o[~gone], out[~gone]) and torch.equal(l[~gone], lse[~gone])
        again, al = s.dense()
        assert torch.equal(again, out) and torch.equal(al, lse)
        ra.ra_paged_check(s.ctx)
    s.done()


def test_what_the_probe_refuses():
    for change in (dict(D=128), dict(page=32), dict(G=9)):
        s = Setup([40], KVH=1, **{**dict(G=2, D=64, page=16), **change})
        q, (o, l) = s.q.to(DEV), s.outputs()
        with pytest.raises(ra.RAError) as e:
            ra.ra_paged_debug_timeout_probe(s.ctx, 0, q.data_ptr(), s.H * s.D, s.D, o.data_ptr(), l.data_ptr(), 1, *s._seqs(), 0, 0, 10 ** 6)
        assert e.value.code == ra.RA_ERR_UNSUPPORTED
        s.done()
    s = Setup([40], KVH=1, G=2, D=64, page=16)
    q, (o, l) = s.q.to(DEV), s.outputs()
    for share, tile, ns in ((0, 0, 10), (0, 0, 10 ** 9), (-1, 0, 10 ** 6), (0, -1, 10 ** 6)):
        with pytest.raises(ra.RAError) as e:
            ra.ra_paged_debug_timeout_probe(s.ctx, 0, q.data_ptr(), 128, 64, o.data_ptr(), l.data_ptr(), 1, *s._seqs(), share, tile, ns)
        assert e.value.code == ra.RA_ERR_INVALID_ARG
    s.done()
