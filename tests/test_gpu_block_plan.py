"""Block plans and trims against the oracle: ids, counters and slots are equal."""
import numpy as np
import pytest
import torch

import paper_2609_29364_amd as nsd
from oracle import prompt
from parity import i32

pytestmark = pytest.mark.gpu


def make(seed, bs, width, n_hi, spare, lens_hi=None, short=False):
    """A batch whose requests hold the blocks of their lengths (some of them more)."""
    rng = np.random.default_rng(seed)
    lens = rng.integers(0, (lens_hi or 16 * width) + 1, bs)
    owned = np.minimum(-(-lens // 16) + rng.integers(0, 3, bs) * (rng.random(bs) < 0.2), width)
    n = np.minimum(rng.integers(0, n_hi + 1, bs), 16 * width - lens if not short else n_hi)
    ids = rng.permutation(int(owned.sum()) + spare).astype(np.int32)
    table = np.full((bs, width), -7, np.int32)
    at = 0
    for r in range(bs):
        table[r, :owned[r]] = ids[at:at + owned[r]]
        at += owned[r]
    indptr = np.concatenate([[0], np.cumsum(n)])
    free = np.concatenate([ids[at:], np.full(13, -5, np.int32)])
    return table, owned, lens, indptr, free, spare


def plan_gpu(dev, table, owned, lens, indptr, free, count, in_place):
    t, o, l, q, f, c = (i32(x, dev) for x in (table, owned, lens, indptr, free, [count]))
    total = int(indptr[-1])
    out = dict(new_owned=o, new_lens=l, new_free_count=c) if in_place else {}
    no, nl, nc, g, s = nsd.plan_blocks(t, o, l, q, f, c, total, **out)
    assert not in_place or (no is o and nl is l and nc is c)
    if not in_place:      # the inputs stay
        assert torch.equal(o, i32(owned, dev)) and torch.equal(l, i32(lens, dev))
        assert c.item() == count
    assert torch.equal(f, i32(free, dev))
    return [x.cpu().numpy() for x in (t, no, nl, nc, g, s)]


CASES = [  # bs, width, new tokens up to, free ids, lengths up to
    (1, 1, 16, 1, 8), (1, 4, 0, 3, None), (1, 600, 9000, 600, 300), (3, 5, 40, 2, None),
    (64, 9, 1, 50, None), (255, 20, 33, 400, None), (1000, 6, 7, 100, None),
    (1025, 10, 40, 0, None), (2049, 30, 20, 3000, None), (8192, 12, 25, 9000, None),
    (8192, 3, 1, 5, None)]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("case", CASES)
def test_plan(device, case, in_place):
    bs, width, n_hi, spare, lens_hi = case
    args = make(bs + width, bs, width, n_hi, spare, lens_hi)
    ref = prompt.plan_blocks(*args, int(args[3][-1]))
    got = plan_gpu(device, *args, in_place)
    for name, a, b in zip(("table", "owned", "lens", "free_count", "granted", "slots"), got, ref):
        assert np.array_equal(a.reshape(-1), np.asarray(b).reshape(-1)), name


def test_plan_leaves_requests_out_that_pass_their_row(device):
    args = make(5, 300, 4, 60, 400, short=True)
    ref = prompt.plan_blocks(*args, int(args[3][-1]))
    assert 0 < ref[4].sum() < 300
    got = plan_gpu(device, *args, False)
    for a, b in zip(got, ref):
        assert np.array_equal(a.reshape(-1), np.asarray(b).reshape(-1))


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("bs, width", [(1, 1), (1, 700), (64, 9), (257, 100), (4096, 33), (8192, 5)])
def test_trim(device, bs, width, in_place):
    rng = np.random.default_rng(bs)
    table, owned, lens, _, free, count = make(bs, bs, width, 0, 7)
    keep = np.where(rng.random(bs) < 0.4, 0, rng.integers(-3, 16 * width + 40, bs))
    free = np.concatenate([free[:count], np.full(max(0, int(owned.sum()) - 2), -5, np.int32)])
    ro, rf, rc = prompt.trim_blocks(table, owned, np.maximum(keep, 0), free, count)
    t, o, k, f, c = (i32(x, device) for x in (table, owned, keep, free, [count]))
    no, nc = nsd.trim_blocks(t, o, k, f, c, **(dict(new_owned=o, new_free_count=c)
                                               if in_place else {}))
    assert np.array_equal(no.cpu().numpy(), ro) and nc.item() == rc
    assert np.array_equal(f.cpu().numpy(), rf) and torch.equal(t, i32(table, device))


def test_rows_behind_the_last_request_have_no_slot(device):
    table, owned, lens, indptr, free, count = make(8, 30, 20, 9, 60, lens_hi=100)
    rt, ro, rl, rc, rg, rs = prompt.plan_blocks(table, owned, lens, indptr, free, count, indptr[-1])
    t, o, l, q, f, c = (i32(x, device) for x in (table, owned, lens, indptr, free, [count]))
    s = nsd.plan_blocks(t, o, l, q, f, c, int(indptr[-1]) + 5000)[4].cpu().numpy()
    assert np.array_equal(s[:indptr[-1]], rs) and (s[indptr[-1]:] == -1).all()
    assert np.array_equal(t.cpu().numpy(), rt)


def test_a_batch_of_none(device):
    e = torch.empty(0, dtype=torch.int32, device=device)
    c = i32([3], device)
    no, nl, nc, g, s = nsd.plan_blocks(e.view(0, 4), e, e, i32([0], device), i32([1, 2, 3], device),
                                       c, 0)
    assert nc.item() == 3 and s.numel() == 0
    no, nc = nsd.trim_blocks(e.view(0, 4), e, e, i32([1, 2, 3], device), c)
    assert nc.item() == 3


def test_contents_out_of_range_stay_in_bounds(device):
    """Counts, lengths, offsets and ids that no valid batch has: whatever comes out, nothing
    beside the outputs changes."""
    bs, width, total = 70, 5, 200
    rng = np.random.default_rng(9)
    wild = lambda n: rng.choice([-2**31, -17, -1, 0, 3, 40, 10**6, 2**31 - 1], n)
    guard = torch.full((bs * width + 64,), -9, dtype=torch.int32, device=device)
    t = guard[32:32 + bs * width].view(bs, width)
    for seed in range(4):
        for f in (nsd.plan_blocks, nsd.trim_blocks):
            o, l, q = i32(wild(bs), device), i32(wild(bs), device), i32(wild(bs + 1), device)
            free, c = i32(wild(20), device), i32([[7, -4, 99, 20][seed]], device)
            if f is nsd.plan_blocks:
                r = f(t, o, l, q, free, c, total)
                assert 0 <= r[2].item() <= 20
                ok = r[4].cpu().numpy()
                assert ((ok >= -1)).all()
            else:
                r = f(t, o, l, free, c)
                assert 0 <= r[1].item() <= 20
            assert (guard[:32] == -9).all() and (guard[-32:] == -9).all()


def test_steps_in_a_graph(device):
    """A captured step updates the state in place: each replay continues from the last."""
    table, owned, lens, _, free, count = make(3, 40, 30, 0, 300, lens_hi=100)
    n = np.full(40, 5)
    indptr = np.concatenate([[0], np.cumsum(n)])
    t, o, l, q, f, c = (i32(x, device) for x in (table, owned, lens, indptr, free, [count]))
    s, g = (torch.empty(k, dtype=torch.int32, device=device) for k in (200, 40))
    first = [x.clone() for x in (t, o, l, c)]

    def step():
        nsd.plan_blocks(t, o, l, q, f, c, 200, new_owned=o, new_lens=l, new_free_count=c,
                        granted=g, slots=s)

    step()
    for x, y in zip((t, o, l, c), first):
        x.copy_(y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    state = (table, owned, lens, indptr, free, count)
    for _ in range(4):
        graph.replay()
        torch.cuda.synchronize()
        rt, ro, rl, rc, rg, rs = prompt.plan_blocks(*state, 200)
        for a, b in ((t, rt), (o, ro), (l, rl), (c, [rc]), (g, rg), (s, rs)):
            assert np.array_equal(a.cpu().numpy(), np.asarray(b))
        state = (rt, ro, rl, indptr, free, rc)
        torch.ones(1000, device=device).sum().item()
