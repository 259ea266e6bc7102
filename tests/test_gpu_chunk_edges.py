"""Chunk attention at the edges of what its call allows, against the oracle under the bounds of
test_gpu_chunk_attention.py."""
import numpy as np
import pytest
import torch

import paper_2609_29364_amd as nsd
from parity import i32
from test_gpu_chunk_attention import Batch, both_sizes

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("indptr, length, hq, hkv, d, max_len", [
    ([0, 1120, 0, 1120], 1024, 32, 8, 128, 1024), ([0, 300] * 128 + [0], 4000, 4, 2, 64, 5000),
    ([0, 2000, 5, 2000, 7, 2000], 9000, 32, 8, 64, 9000)])
def test_offsets_that_fall_stay_in_bounds(device, indptr, length, hq, hkv, d, max_len):
    """Offsets that count the same rows over and over: more items than the host can know of
    (test_chunk_plan.py counts them).  Nothing beside the output and the workspace changes, and
    every row of the output is a request's or untouched."""
    bs, total, nb = len(indptr) - 1, max(indptr), 600
    g = torch.Generator().manual_seed(bs)
    bf = lambda *s: torch.randn(s, generator=g).bfloat16().to(device)
    q, k, v = bf(total, hq, d), bf(nb, hkv, d // 8, 16, 8), bf(nb, hkv, d, 16)
    table = torch.randint(0, nb, (bs, -(-length // 16)), generator=g, dtype=torch.int32).to(device)
    need = nsd.chunk_attention_workspace_size(bs, total, hq, hkv, d, total, max_len)
    for fill in (0, 255, 1):
        room = torch.full((need + 512,), fill, dtype=torch.uint8, device=device)
        out = torch.full((total + 64, hq, d), 7.0, dtype=torch.bfloat16, device=device)
        nsd.chunk_attention(q, k, v, table, i32([length] * bs, device), i32(indptr, device), total,
                            max_len, out=out[32:-32], workspace=room[256:256 + need])
        torch.cuda.synchronize()
        assert (out[:32] == 7).all() and (out[-32:] == 7).all()
        assert (room[:256] == fill).all() and (room[256 + need:] == fill).all()
        # averages of V, or untouched
        assert torch.isfinite(out).all() and out.abs().max() <= 7


@both_sizes
@pytest.mark.parametrize("slopes", [None, [0.0, 0.05, 0.003, 0.2]])
def test_rows_before_position_0_see_the_prefix(device, slopes, bound):
    """Requests shorter than their new tokens: whole waves of rows before position 0, and waves
    that hold rows of both kinds."""
    b = Batch(device, [0, 0, 0], [300, 90, 70], 4, 2, 64)
    b.lens = [40, 20, 64]
    b.kv = [[x[:n] for x in kv] for kv, n in zip(b.kv, b.lens)]
    prefix = [33, 70, 0]
    kw = dict(prefix=prefix) if slopes is None else dict(prefix=prefix, slopes=slopes)
    got = b.run(bound=bound, **kw).double().cpu().numpy()
    ref, tol = b.ref(**kw)
    # distances reach 300, past the lengths that the bound takes
    tol = tol + 2.0**-21 * (0.2 * 300 if slopes else 0) * 5
    assert (np.abs(got - ref) <= tol).all()
    assert (np.abs(got[:260]).max((1, 2)) > 0).all()      # the prefix alone
    assert (got[390:396] == 0).all()                      # no prefix: nothing


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("slopes", [None, [0.25, 1.0, 0.0, -0.01]])
@pytest.mark.parametrize("softcap, scale", [(200.0, None), (256.0, None), (257.0, None), (1e3, None),
                                            (3e4, -0.2), (1e6, None), (1e8, None), (3e38, None),
                                            (300.0, 8.0), (1e4, 300.0), (1e4, -1000.0)])
def test_large_caps(device, softcap, scale, slopes, d):
    """A cap far above the scores leaves them alone, one among large scores bends them.

    A capped score is off by a few 2^-23 of itself where it is formed, and from the product by what
    the scale makes of 128 * 2^-24 * sum |q k|: both in a weight and in the maximum."""
    b = Batch(device, [0, 130, 300], [70, 1, 40], 4, 2, d)
    ref, tol = b.ref(scale=scale, softcap=softcap, slopes=slopes)
    v = np.abs(np.concatenate([x[1].float().numpy().reshape(-1) for x in b.kv])).max()
    top = min(softcap, abs(scale or d ** -0.5) * 6 * d)
    product = abs(scale or d ** -0.5) * 128 * 2.0**-24 * 2 * d
    tol = tol + 2 * (8 * 2.0**-23 * top + product) * v
    for bound in (0, 5000):
        got = b.run(scale=scale, softcap=softcap, slopes=slopes, bound=bound).double().cpu().numpy()
        assert (np.abs(got - ref) <= tol).all()


@pytest.mark.parametrize("bs", [300, 256])
def test_capped_single_tokens_of_many_requests(device, bs):
    rng = np.random.default_rng(bs)
    b = Batch(device, rng.integers(0, 200, bs).tolist(), [1] * bs, 4, 2, 64)
    b.check(softcap=5.0)
    b.check(softcap=1e5)


@pytest.mark.parametrize("length, every, nth", [(1500, 2, 1), (4096, 4, 1), (4096, 4, 3), (4096, 1, 0),
                                                (4096, 16, 7)])
def test_parts_of_nan_scores_reach_the_row(device, length, every, nth):
    """A split context of which every so many parts (256 tokens each) have no score but NaN."""
    b = Batch(device, [length - 1], [1], 4, 2, 64)
    for t in range(length):
        if t // 256 % every == nth:
            b.put(0, t, k=float("nan"))
    assert torch.isnan(b.run(bound=length)).all()


@both_sizes
@pytest.mark.parametrize("softcap", [0.0, 20.0])
@pytest.mark.parametrize("scale", [3e38, -3e38])
def test_the_largest_scale(device, scale, softcap, bound):
    b = Batch(device, [40], [50], 2, 1, 64)
    b.q.zero_()
    got = b.run(scale=scale, softcap=softcap, bound=bound).double().cpu().numpy()
    ref, tol = b.ref(scale=0.0)                           # every score is 0
    assert (np.abs(got - ref) <= tol).all()


@pytest.mark.parametrize("hkv", [513, 1024, 1025, 2050])
def test_more_heads_than_workgroups_at_once(device, hkv):
    b = Batch(device, [40, 0], [1, 18], hkv, hkv, 64)
    b.check()
    b.check(b.run(bound=10000))


def test_one_long_context_among_many_items(device):
    """More (item, KV head) pairs than two rounds take, with one context far longer than the rest,
    past the lengths up to which such batches are not split."""
    bs = 140
    rng = np.random.default_rng(1)
    ctx, new = rng.integers(0, 60, bs), np.ones(bs, int)
    ctx[77], new[3] = 9000, 90
    b = Batch(device, ctx.tolist(), new.tolist(), 16, 8, 64)
    assert nsd.chunk_attention_workspace_size(bs, b.total, 16, 8, 64, 90, max(b.lens)) > 0
    b.check(b.run())
    pos = np.concatenate([np.arange(c, c + n) for c, n in zip(b.ctx, b.new)])
    kw = dict(first=np.maximum(pos - 8000, 0), prefix=[20] * bs, softcap=30.0)
    b.check(b.run(**kw), **kw)


def test_one_workspace_for_batches_of_any_size(device):
    ws = nsd.new_workspace(nsd.chunk_attention_workspace_bound(8, 64), device)
    rng = np.random.default_rng(2)
    for bs, hi in ((256, 300), (100, 900), (7, 2000), (1, 4000), (30, 1200)):
        new = np.ones(bs, int)
        new[0] = 20
        b = Batch(device, rng.integers(0, hi, bs).tolist(), new.tolist(), 16, 8, 64, seed=bs)
        b.check([b.run(bound=4096, workspace=ws), b.run(bound=100000, workspace=ws)])
