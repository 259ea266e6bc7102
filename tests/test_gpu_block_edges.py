"""Block plans at the edges of what their call allows, against the oracle."""
import numpy as np
import pytest
import torch

import paper_2609_29364_amd as nsd
from oracle import prompt
from parity import i32
from test_gpu_block_plan import make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ahead", [1, 5, 40, 5000])
def test_rows_ahead_of_the_first_request_have_no_slot(device, ahead):
    """Offsets that do not begin at 0: the rows before them are no request's, and a slot of theirs
    would be one of the first request's cached tokens."""
    table, owned, lens, indptr, free, count = make(8, 30, 20, 9, 60, lens_hi=100)
    lens[0], owned[0] = 100, 20
    table[0] = np.arange(500, 520)
    indptr = indptr + ahead
    rt, ro, rl, rc, rg, rs = prompt.plan_blocks(table, owned, lens, indptr, free, count, indptr[-1])
    assert (rs[:ahead] == -1).all() and (rs[ahead:] >= 0).any()
    t, o, l, q, f, c = (i32(x, device) for x in (table, owned, lens, indptr, free, [count]))
    no, nl, nc, g, s = nsd.plan_blocks(t, o, l, q, f, c, int(indptr[-1]))
    for a, b in ((t, rt), (no, ro), (nl, rl), (nc, [rc]), (g, rg), (s, rs)):
        assert np.array_equal(a.cpu().numpy(), np.asarray(b))


@pytest.mark.parametrize("total", [1, 37, 9000])
def test_rows_of_a_batch_of_none_have_no_slot(device, total):
    e = torch.empty(0, dtype=torch.int32, device=device)
    s = torch.full((total + 2,), 5, dtype=torch.int32, device=device)
    out = nsd.plan_blocks(e.view(0, 4), e, e, i32([0], device), i32([1, 2, 3], device),
                          i32([3], device), total, slots=s[1:-1])
    assert out[2].item() == 3
    assert (out[4] == -1).all() and s[0].item() == 5 and s[-1].item() == 5


def test_lengths_past_31_bits_are_not_granted(device):
    """A table row with room for more tokens than a length counts."""
    width = 2**27 + 8
    table = torch.zeros((1, width), dtype=torch.int32, device=device)
    for length, n, ok in ((2**31 - 20, 19, 1), (2**31 - 20, 20, 0), (2**31 - 1, 100, 0)):
        no, nl, nc, g, s = nsd.plan_blocks(table, i32([width], device), i32([length], device),
                                           i32([0, n], device), i32([1, 2, 3], device),
                                           i32([3], device), n)
        assert g.item() == ok and nl.item() == length + n * ok and nc.item() == 3
        assert no.item() == width
        assert ((s >= 0) if ok else (s == -1)).all()
