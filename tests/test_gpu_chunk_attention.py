"""Attention of a chunk over the paged cache against the oracle.

With w the softmax weights, an output is within
    2^-8 |o| + (2^-8 + 3e-4 + 2^-21 max|y|) sum w |v| + 1e-6
of the 64-bit value: half a step of its own rounding, half a step of each weight's rounding to
bf16, the fp32 product's error over a head (at most 128 * 2^-24 * sum |q k| scale < 1e-4 at these
values, in the weight and in their sum) and exponent (2^-23 of y, in a weight and in the maximum).
"""
import numpy as np
import pytest
import torch

import paper_2609_29364_amd as nsd
from oracle import prompt
from parity import i32

pytestmark = pytest.mark.gpu
LONG = 5000     # a bound of the lengths for which items have 128 rows
both_sizes = pytest.mark.parametrize("bound", [0, LONG])


class Batch:
    """Requests of `new` tokens after `ctx` cached ones; the pool's other slots hold NaN."""

    def __init__(self, dev, ctx, new, hq=4, hkv=2, d=64, seed=0, spare=3, width=0):
        self.dev, self.ctx, self.new = dev, ctx, new
        self.hq, self.hkv, self.d = hq, hkv, d
        rng = np.random.default_rng(seed)
        g = torch.Generator().manual_seed(seed)
        self.lens = [c + n for c, n in zip(ctx, new)]
        self.indptr = np.concatenate([[0], np.cumsum(new)]).astype(int)
        self.total = int(self.indptr[-1])
        counts = [-(-n // 16) for n in self.lens]
        nb = sum(counts) + spare
        ids = rng.permutation(nb)
        self.table = np.full((len(ctx), max(1, width, *counts)), -1, np.int32)
        self.k = torch.full((nb, hkv, d // 8, 16, 8), float("nan")).bfloat16()
        self.v = torch.full((nb, hkv, d, 16), float("nan")).bfloat16()
        self.q = torch.randn((self.total, hq, d), generator=g).bfloat16()
        self.kv = []
        at = 0
        for r, n in enumerate(self.lens):
            k, v = (torch.randn((n, hkv, d), generator=g).bfloat16() for _ in range(2))
            mine = torch.from_numpy(ids[at:at + counts[r]])
            at += counts[r]
            self.table[r, :counts[r]] = mine.numpy()
            self.kv.append([k, v])
            t = torch.arange(n)
            self.k[mine[t // 16], :, :, t % 16] = k.view(n, hkv, d // 8, 8)
            self.v[mine[t // 16], :, :, t % 16] = v
        self.nb = nb

    def put(self, r, t, k=None, v=None):
        """Token t of request r gets these values."""
        b = int(self.table[r, t // 16])
        if k is not None:
            self.kv[r][0][t] = k
            self.k[b, :, :, t % 16] = self.kv[r][0][t].view(self.hkv, -1, 8)
        if v is not None:
            self.kv[r][1][t] = v
            self.v[b, :, :, t % 16] = self.kv[r][1][t]

    def run(self, first=None, prefix=None, slopes=None, bound=0, **kw):
        """bound: max_seq_len at least; a long one has items of 128 rows, which a short batch's
        own lengths would not."""
        dev = self.dev
        kw = dict(kw, first_keys=None if first is None else i32(first, dev),
                  prefix_lens=None if prefix is None else i32(prefix, dev),
                  slopes=None if slopes is None else torch.tensor(slopes, dtype=torch.float32,
                                                                  device=dev))
        out = torch.full(self.q.shape, 7.0, dtype=torch.bfloat16, device=dev)
        return nsd.chunk_attention(self.q.to(dev), self.k.to(dev), self.v.to(dev),
                                   i32(self.table, dev), i32(self.lens, dev), i32(self.indptr, dev),
                                   max(1, *self.new), max(1, bound, *self.lens), out=out, **kw)

    def ref(self, scale=None, softcap=0.0, slopes=None, first=None, prefix=None, valid=None):
        """(outputs, bounds), [total_q][Hq][D]."""
        out, tol = [], []
        scale = 1 / np.sqrt(self.d) if scale is None else scale
        for r in range(len(self.new)):
            a, b = self.indptr[r], self.indptr[r + 1]
            k, v = (x.double().numpy() for x in self.kv[r])
            q = self.q[a:b].double().numpy()
            o = prompt.chunk_attention_request(
                q, k, np.concatenate([v, np.abs(v)], -1), self.lens[r], scale, softcap, slopes,
                None if first is None else first[a:b], 0 if prefix is None else prefix[r],
                None if valid is None else valid[r])
            o, size = o[..., :self.d], o[..., self.d:]
            y = abs(scale) * np.sqrt(self.d) * 40 + (0 if slopes is None else
                                                     max(np.abs(slopes)) * self.lens[r])
            out.append(o)
            tol.append(2.0**-8 * np.abs(o) + (2.0**-8 + 3e-4 + 2.0**-21 * y) * size + 1e-6)
        return np.concatenate(out), np.concatenate(tol)

    def check(self, got=None, rows=None, **kw):
        if got is None:
            valid = kw.pop("valid", None)
            got = [self.run(**kw), self.run(bound=LONG, **kw)]
            kw["valid"] = valid
        ref, tol = self.ref(**kw)
        rows = slice(None) if rows is None else rows
        for x in got if isinstance(got, list) else [got]:
            x = x.double().cpu().numpy()
            with np.errstate(invalid="ignore"):
                err = np.abs(x - ref)
            assert np.isfinite(x[rows]).all()
            assert (err[rows] <= tol[rows]).all(), \
                f"{float((err - tol)[rows].max())} past the bound, rows {np.unique(np.argwhere(err > tol)[:, 0])[:9]}"


@pytest.mark.parametrize("hq, hkv, d", [(4, 2, 64), (32, 8, 128), (16, 8, 128), (8, 8, 64), (5, 1, 128),
                                        (12, 4, 64), (7, 7, 128), (40, 1, 64)])
def test_heads(device, hq, hkv, d):
    Batch(device, [0, 33, 100, 7], [40, 1, 70, 16], hq, hkv, d).check()


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 200])
@pytest.mark.parametrize("ctx", [0, 1, 47])
def test_lengths(device, n, ctx):
    Batch(device, [ctx], [n], 8, 2, 128, seed=n).check()


def test_requests_without_new_tokens(device):
    b = Batch(device, [5, 0, 70, 20, 9], [0, 0, 33, 0, 4])
    b.check()
    Batch(device, [64], [0]).run()


@pytest.mark.parametrize("bs", [63, 64, 65, 300])
def test_many_requests(device, bs):
    rng = np.random.default_rng(bs)
    new = rng.choice([0, 1, 1, 1, 5, 40], bs).tolist()
    Batch(device, rng.integers(0, 90, bs).tolist(), new, 4, 2, 64, seed=bs).check()


def test_the_largest_batch(device):
    Batch(device, [3] * 8192, [1] * 8192, 2, 1, 64).check()


@pytest.mark.parametrize("ctx, new", [([2000], [1]), ([1500, 3], [5, 1]), ([4095], [1]), ([900], [300]),
                                      ([0, 2500], [1, 30])])
def test_split_contexts(device, ctx, new):
    b = Batch(device, ctx, new, 4, 2, 128)
    assert nsd.chunk_attention_workspace_size(len(ctx), b.total, 4, 2, 128, max(new),
                                              max(b.lens)) > 0
    b.check()
    # the batch with room for much longer contexts takes more splits, some of them empty
    dev = device
    out = nsd.chunk_attention(b.q.to(dev), b.k.to(dev), b.v.to(dev), i32(b.table, dev),
                              i32(b.lens, dev), i32(b.indptr, dev), max(new), 100000)
    b.check(out)


@pytest.mark.parametrize("options", [{}, dict(softcap=20.0, slopes=[0.5, 0.01, 0.0, 0.002] * 2)])
def test_long_chunks(device, options):
    b = Batch(device, [3000, 1200, 40], [300, 129, 1], 8, 2, 128)
    b.check(**options)
    pos = np.concatenate([np.arange(c, c + n) for c, n in zip(b.ctx, b.new)])
    b.check(first=np.maximum(pos - 700, 0), prefix=[200, 0, 3], **options)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("ctx, new", [([2500], [1]), ([1500, 20], [3, 40]), ([1100, 900, 30], [70, 1, 2])])
def test_split_contexts_with_masks(device, ctx, new, d):
    b = Batch(device, ctx, new, 4, 2, d, seed=d)
    assert nsd.chunk_attention_workspace_size(len(ctx), b.total, 4, 2, d, max(new), max(b.lens)) > 0
    pos = np.concatenate([np.arange(c, c + n) for c, n in zip(b.ctx, b.new)])
    b.check(first=np.maximum(pos - 1000, 0), prefix=[70] * len(ctx), softcap=8.0,
            slopes=[0.5, 0.002, 0.0, 0.01])
    # a split that sees nothing, and infinities in hidden tokens of others
    first = np.maximum(pos - 5, 0)
    b.put(0, 50, k=float("nan"), v=float("inf"))
    b.put(0, 700, v=float("nan"))
    b.check(first=first)


@pytest.mark.parametrize("bs, hkv, ctx_hi", [(20, 32, 60), (70, 8, 900), (130, 4, 1500), (256, 2, 800),
                                             (257, 4, 100)])
def test_batches_placed_by_length(device, bs, hkv, ctx_hi):
    """Batches whose items are ordered, and split, by the lengths of one to four requests a lane."""
    rng = np.random.default_rng(bs)
    ctx = np.where(rng.random(bs) < 0.8, rng.integers(0, 60, bs), rng.integers(0, ctx_hi, bs))
    new = rng.choice([0, 1, 1, 1, 1, 2, 40], bs)
    new[rng.integers(bs)] = 130
    Batch(device, ctx.tolist(), new.tolist(), 2 * hkv, hkv, 64, seed=bs).check()


@pytest.mark.parametrize("ctx, new", [([600], [272]), ([300, 500], [200, 90])])
def test_a_last_round_of_few_items(device, ctx, new):
    """17 to 19 items where 16 run at once: those of the last round are split."""
    b = Batch(device, ctx, new, 256, 32, 64)
    pos = np.concatenate([np.arange(c, c + n) for c, n in zip(b.ctx, b.new)])
    b.check(first=np.maximum(pos - 400, 0), prefix=[30] * len(ctx))


def test_rows_behind_the_last_request_stay(device):
    b = Batch(device, [30, 500, 2], [20, 1, 7], 4, 2, 64)
    dev, pad = device, 300
    q = torch.cat([b.q, torch.randn((pad, 4, 64)).bfloat16()]).to(dev)
    out = torch.full_like(q, 7.0)
    nsd.chunk_attention(q, b.k.to(dev), b.v.to(dev), i32(b.table, dev), i32(b.lens, dev),
                        i32(b.indptr, dev), 20, 501, out=out)
    b.check(out[:b.total])
    assert (out[b.total:] == 7).all()


def test_a_tiny_cap(device):
    b = Batch(device, [40], [50], 2, 1, 64)
    got = b.run(softcap=1e-38).double().cpu().numpy()     # every score is then 0
    ref, tol = b.ref(scale=0.0)
    assert (np.abs(got - ref) <= tol).all()


@pytest.mark.parametrize("scale", [0.0, -0.2, 1.0, 1e-3])
def test_scales(device, scale):
    Batch(device, [50, 0], [70, 3], 4, 2, 64).check(scale=scale)


OPTIONS = [dict(softcap=5.0), dict(softcap=50.0, scale=-0.3), dict(slopes=[0.0, 0.5, 0.03, 2.0]),
           dict(softcap=20.0, slopes=[0.25, 1.0, 0.0, -0.01])]


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("options", OPTIONS)
def test_caps_and_slopes(device, options, d, masked):
    b = Batch(device, [0, 130, 300, 2], [70, 1, 150, 30], 4, 2, d)
    if masked:
        rng = np.random.default_rng(1)
        pos = np.concatenate([np.arange(c, c + n) for c, n in zip(b.ctx, b.new)])
        options = dict(options, first=np.maximum(pos - rng.integers(0, 200, len(pos)), 0),
                       prefix=[3, 0, 64, 32])
    b.check(**options)


@pytest.mark.parametrize("window", [1, 2, 16, 63, 64, 65, 100])
@pytest.mark.parametrize("prefix", [0, 1, 64, 100])
def test_windows(device, window, prefix):
    b = Batch(device, [0, 200, 333], [150, 1, 65], 8, 2, 64, seed=window)
    pos = np.concatenate([np.arange(c, c + n) for c, n in zip(b.ctx, b.new)])
    b.check(first=np.maximum(pos - window + 1, 0), prefix=[prefix] * 3)


def test_documents(device):
    b = Batch(device, [40, 0], [300, 100], 4, 2, 128)
    starts = [0, 17, 60, 61, 200, 330]
    pos = [np.arange(c, c + n) for c, n in zip(b.ctx, b.new)]
    first = [np.array(starts)[np.searchsorted(starts, p, side="right") - 1] for p in pos]
    b.check(first=np.concatenate(first))


def test_prefixes_ahead_of_their_queries(device):
    # every query sees the prefix, also the part after it; lengths past the request are clamped
    b = Batch(device, [0, 10, 0, 0], [100, 200, 50, 1], 4, 2, 64)
    b.check(prefix=[100, 150, 0, 1])
    got = b.run(prefix=[100, 150, -5, 2**31 - 1])
    b.check(got, prefix=[100, 150, 0, 1])


@both_sizes
def test_rows_that_see_nothing(device, bound):
    b = Batch(device, [0, 100, 50], [80, 3, 70], 4, 2, 128)
    first = np.full(b.total, 0)
    first[5:60] = 10**6
    first[83:100] = 2**31 - 1
    first[100:110] = -2**31
    got = b.run(first=first, bound=bound)
    b.check(got, first=first)
    assert (got[5:60] == 0).all() and (got[83:100] == 0).all()
    # nothing at all for whole workgroups
    assert (b.run(first=np.full(b.total, 10**6), bound=bound) == 0).all()


@both_sizes
def test_lengths_shorter_than_the_new_tokens(device, bound):
    b = Batch(device, [0, 0], [90, 20], 4, 2, 64)
    b.lens = [50, 0]
    b.kv = [[x[:50] for x in b.kv[0]], [x[:1] for x in b.kv[1]]]
    got = b.run(bound=bound)
    ref, tol = prompt.chunk_attention_request(
        b.q[:90].double().numpy(), *(x.double().numpy() for x in b.kv[0]), 50, 0.125), 0.05
    assert (got[:40] == 0).all() and (got[90:] == 0).all()
    assert (np.abs(got[:90].double().cpu().numpy() - ref) <= tol).all()


@pytest.mark.parametrize("what", ["k", "v", "both"])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_infinities_and_nan_in_hidden_tokens(device, value, what):
    """A hidden token's K and V do not reach the rows that it is hidden from."""
    b = Batch(device, [20, 90], [120, 2], 4, 2, 64)
    pos = np.concatenate([np.arange(20, 140), [90, 91]])
    first = np.maximum(pos - 29, 0)
    hidden = {0: (0, 1, 77, 139), 1: (0, 40, 61)}
    for r, ts in hidden.items():
        for t in ts:
            b.put(r, t, k=value if what != "v" else None, v=value if what != "k" else None)
    rows = [i for i, p in enumerate(pos) if not any(
        p - 29 <= t <= p for t in hidden[0 if i < 120 else 1])]
    assert 50 < len(rows) < 122
    b.check(first=first, rows=rows)


@both_sizes
def test_infinite_values_reach_the_rows_that_see_them(device, bound):
    b = Batch(device, [10], [60], 2, 1, 64)
    inf, nan = float("inf"), float("nan")
    v = b.kv[0][1]
    for t, dim, x in ((30, 3, inf), (31, 4, -inf), (32, 5, nan), (33, 3, -inf)):
        row = v[t].clone()
        row[0, dim] = x
        b.put(0, t, v=row)
    got = b.run(bound=bound).float().cpu()
    at = lambda p, dim: got[p - 10, 0, dim]
    assert torch.isfinite(got[:20]).all()
    assert at(30, 3) == inf and at(32, 3) == inf and torch.isnan(at(33, 3)) and torch.isnan(at(69, 3))
    assert at(31, 4) == -inf and at(69, 4) == -inf and torch.isnan(at(32, 5))
    others = [i for i in range(64) if i not in (3, 4, 5)]
    assert torch.isfinite(got[..., others]).all()


def test_blocks_that_cannot_be_read(device):
    b = Batch(device, [300, 0, 64], [40, 50, 1], 4, 2, 64)
    valid = [np.ones(n, bool) for n in b.lens]
    for r, blk, i in ((0, 0, -1), (0, 5, b.nb), (0, 20, 2**31 - 1), (1, 1, -2**31), (2, 4, -1)):
        b.table[r, blk] = i
        valid[r][blk * 16:(blk + 1) * 16] = False
    b.check(valid=valid)
    # a request none of whose blocks is valid, and a pool without blocks
    b.table[1] = -1
    for bound in (0, LONG):
        assert (b.run(bound=bound)[40:90] == 0).all()
    e = torch.empty((0, 2, 8, 16, 8), dtype=torch.bfloat16, device=device)
    out = nsd.chunk_attention(b.q.to(device), e, e.view(0, 2, 64, 16), i32(b.table, device),
                              i32(b.lens, device), i32(b.indptr, device), 50, 400)
    assert (out == 0).all()


def test_offsets_and_lengths_out_of_range_stay_in_bounds(device):
    b = Batch(device, [30] * 70, [2] * 70, 4, 2, 64)
    rng = np.random.default_rng(0)
    wild = lambda n: rng.choice([-2**31, -5, 0, 1, 60, 139, 140, 10**6, 2**31 - 1], n)
    room = torch.full((b.total + 16, 4, 64), 7.0, dtype=torch.bfloat16, device=device)
    for _ in range(4):
        nsd.chunk_attention(b.q.to(device), b.k.nan_to_num().to(device),
                            b.v.nan_to_num().to(device), i32(wild(b.table.shape), device),
                            i32(wild(70), device), i32(wild(71), device), 2, 64,
                            first_keys=i32(wild(b.total), device),
                            prefix_lens=i32(wild(70), device), out=room[8:-8])
        nsd.chunk_attention(b.q.to(device), b.k.nan_to_num().to(device),
                            b.v.nan_to_num().to(device), i32(wild(b.table.shape), device),
                            i32(wild(70), device), i32(wild(71), device), 2, LONG,
                            first_keys=i32(wild(b.total), device),
                            prefix_lens=i32(wild(70), device), out=room[8:-8])
        assert (room[:8] == 7).all() and (room[-8:] == 7).all()


@both_sizes
def test_large_scores(device, bound):
    """Scores of some thousand, growing along the context: the maximum moves on and on."""
    b = Batch(device, [500], [33], 2, 1, 128)
    for t in range(533):
        b.put(0, t, k=b.kv[0][0][t] * (1 + t / 8))
    got = b.run(scale=1.0, bound=bound).double().cpu().numpy()
    ref, _ = b.ref(scale=1.0)
    # the weights' exponents carry 2^-24 of scores up to about 3e3 in each of some roundings
    size = np.abs(b.kv[0][1].double().numpy()).max()
    assert np.abs(got - ref).max() <= 2.0**-8 * size + 128 * 2.0**-24 * 3e3 * 4 * size


def test_agrees_with_verification(device):
    b = Batch(device, [1000, 30, 517, 64], [5, 5, 1, 3], 32, 8, 128)
    args = [x.to(device) for x in (b.q, b.k, b.v)] + [i32(x, device) for x in
                                                      (b.table, b.lens, b.indptr)]
    a = nsd.chunk_attention(*args, 5, 1005)
    c = nsd.verify_attention(*args, 5, 1005)
    assert (a.float() - c.float()).abs().max() <= 2e-2


def test_a_pool_past_32_bits(device):
    """Block ids whose byte offsets pass 2^32 and element offsets 2^31."""
    nb, hkv, d = 140000, 8, 128
    k = torch.zeros((nb, hkv, d // 8, 16, 8), dtype=torch.bfloat16, device=device)
    v = torch.zeros((nb, hkv, d, 16), dtype=torch.bfloat16, device=device)
    b = Batch(device, [70], [40], 32, 8, 128, spare=0)
    ids = torch.tensor([nb - 1, 131072, 0, 65536, nb - 2, 70000, 139000])
    k[ids.to(device)] = b.k[torch.from_numpy(b.table[0]).long()].to(device)
    v[ids.to(device)] = b.v[torch.from_numpy(b.table[0]).long()].to(device)
    b.table[0] = ids.numpy()
    out = nsd.chunk_attention(b.q.to(device), k, v, i32(b.table, device), i32(b.lens, device),
                              i32(b.indptr, device), 40, 110)
    b.check(out)
    # and through rope_append into them
    slots = np.concatenate([b.table[0][np.arange(70, 110) // 16].astype(np.int64) * 16
                            + np.arange(70, 110) % 16])
    rows = [x[70:].to(device) for x in b.kv[0]]
    k[ids.to(device)[4:]] = 0
    v[ids.to(device)[4:]] = 0
    for t in range(64, 70):
        k[int(ids[4]), :, :, t % 16] = b.kv[0][0][t].view(8, 16, 8).to(device)
        v[int(ids[4]), :, :, t % 16] = b.kv[0][1][t].to(device)
    q = nsd.rope_append(k, v, b.q.to(device), *rows, torch.zeros(40, dtype=torch.int32, device=device),
                        torch.ones(64, device=device), i32(slots, device))
    assert torch.equal(q.cpu(), b.q)
    again = nsd.chunk_attention(q, k, v, i32(b.table, device), i32(b.lens, device),
                                i32(b.indptr, device), 40, 110)
    assert torch.equal(again, out)


def test_streams_and_repeats(device):
    """The same bits on another stream, with a new workspace and in any company."""
    b = Batch(device, [700, 20, 3], [30, 200, 1], 8, 2, 128)
    args = [x.to(device) for x in (b.q, b.k, b.v)] + [i32(x, device) for x in
                                                      (b.table, b.lens, b.indptr)]
    a = nsd.chunk_attention(*args, 200, 730)
    need = nsd.chunk_attention_workspace_size(3, b.total, 8, 2, 128, 200, 730)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(device) for _ in range(3)]
    outs = []
    for s in streams:
        with torch.cuda.stream(s):
            for _ in range(5):
                ws = torch.full((need + 64,), 255, dtype=torch.uint8, device=device)
                outs.append(nsd.chunk_attention(*args, 200, 730, workspace=ws))
    torch.cuda.synchronize()
    assert all(torch.equal(o, a) for o in outs)


def test_refusals(device):
    b = Batch(device, [20], [5], 4, 2, 64)
    args = dict(q=b.q.to(device), k=b.k.to(device), v=b.v.to(device), t=i32(b.table, device),
                l=i32(b.lens, device), i=i32(b.indptr, device), mq=5, ml=25)
    call = lambda kw={}, **bad: nsd.chunk_attention(*[bad.get(n, x) for n, x in args.items()], **kw)
    call()
    for bad in (dict(k=args["k"][:, :1]), dict(t=args["t"][0]), dict(i=args["i"][:1]),
                dict(q=args["q"].transpose(0, 1)), dict(q=args["q"].cpu())):
        with pytest.raises(ValueError):
            call(**bad)
    with pytest.raises(TypeError):
        call(q=args["q"].half())
    for kw in (dict(first_keys=args["l"]), dict(prefix_lens=args["i"]),
               dict(slopes=torch.ones(3, device=device)), dict(out=args["q"][:3])):
        with pytest.raises(ValueError):
            call(kw)
    for kw in (dict(softcap=-1.0), dict(scale=float("nan"))):
        with pytest.raises(nsd.NsdError):
            call(kw)
    with pytest.raises(nsd.NsdError, match="workspace"):
        call(dict(workspace=torch.empty(16, dtype=torch.uint8, device=device)), ml=32768)
