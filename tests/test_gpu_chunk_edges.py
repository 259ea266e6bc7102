"""Chunk attention at the edges of what its call allows."""
import pytest
import torch

import paper_2609_29364_amd as nsd
from parity import i32

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
