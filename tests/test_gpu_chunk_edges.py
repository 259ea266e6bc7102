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
