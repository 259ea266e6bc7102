"""Prompts through the prompt path as a worker runs it: chunk after chunk beside single tokens,
over two layers, then a verification round on the cache that it left."""
import numpy as np
import pytest
import torch

import paper_2609_29364_amd as nsd
from oracle import prompt
from paper_2609_29364_amd.round import prefill_chunk
from parity import i32

pytestmark = pytest.mark.gpu

HQ, HKV, D, LAYERS, POOL, WIDTH = 8, 2, 64, 2, 64, 40


class Worker:
    def __init__(self, dev, bs, seed=0):
        self.dev, self.bs = dev, bs
        self.gen = torch.Generator().manual_seed(seed)
        zeros = lambda *s: torch.full(s, float("nan"), dtype=torch.bfloat16, device=dev)
        self.k, self.v = zeros(LAYERS, POOL, HKV, D // 8, 16, 8), zeros(LAYERS, POOL, HKV, D, 16)
        rng = np.random.default_rng(seed)
        self.free = i32(rng.permutation(POOL), dev)
        self.count = i32([POOL], dev)
        self.table = i32(np.full((bs, WIDTH), -1), dev)
        self.owned, self.lens = i32([0] * bs, dev), i32([0] * bs, dev)
        self.freq = torch.tensor(1e4 ** (-np.arange(D // 2) / (D // 2)), dtype=torch.float32)
        self.host = [[[], []] for _ in range(bs * LAYERS)]      # turned K rows and V rows
        self.len = [0] * bs

    def rows(self, n):
        return [tuple(torch.randn((n, h, D), generator=self.gen).bfloat16() for h in (HQ, HKV, HKV))
                for _ in range(LAYERS)]

    def step(self, new, granted=None, **kw):
        indptr = np.concatenate([[0], np.cumsum(new)]).astype(int)
        pos = np.concatenate([np.arange(l, l + n) for l, n in zip(self.len, new)] + [np.zeros(0, int)])
        rows = self.rows(indptr[-1])
        outs, g, slots = prefill_chunk(
            self.k, self.v, [tuple(t.to(self.dev) for t in r) for r in rows], i32(pos, self.dev),
            self.freq.to(self.dev), self.table, self.owned, self.lens, i32(indptr, self.dev),
            self.free, self.count, int(indptr[-1]), max(1, *new), 16 * WIDTH, **kw)
        expect = granted or [1] * self.bs
        assert g.tolist() == expect
        for r in range(self.bs):
            if expect[r]:
                self.len[r] += new[r]
        assert self.lens.tolist() == self.len
        for layer in range(LAYERS):
            q, k, v = (t.double().numpy() for t in rows[layer])
            q, k = (torch.from_numpy(prompt.rotate(x, pos, self.freq.numpy())).bfloat16().double()
                    .numpy() for x in (q, k))
            got = outs[layer].double().cpu().numpy()
            for r in range(self.bs):
                a, b = indptr[r], indptr[r + 1]
                if not expect[r]:
                    continue
                h = self.host[r * LAYERS + layer]
                h[0].append(k[a:b])
                h[1].append(v[a:b])
                if a == b:
                    continue
                kk, vv = np.concatenate(h[0]), np.concatenate(h[1])
                ref = prompt.chunk_attention_request(q[a:b], kk, vv, self.len[r], D ** -0.5,
                                                     kw.get("softcap", 0.0))
                # q and k rounded the other way beside a tie move a score by up to 2^-8 of its
                # sum of |q k|, at most 2^-8 * 80 / 8; the weights by that, outputs by theirs
                assert np.abs(got[a:b] - ref).max() <= 0.05
        return outs


def test_chunks_and_single_tokens(device):
    w = Worker(device, 3)
    for new in ([50, 1, 0], [33, 1, 100], [1, 1, 64], [1, 70, 1], [0, 0, 0], [1, 1, 1]):
        w.step(new)
    w.step([20, 1, 2], softcap=10.0)
    used = sum(-(-n // 16) for n in w.len)
    assert w.count.item() == POOL - used
    # a verification round's attention reads the same cache
    q = torch.randn((3, HQ, D), generator=w.gen).bfloat16()
    got = nsd.verify_attention(q.to(device), w.k[1], w.v[1], w.table, w.lens, i32([0, 1, 2, 3], device),
                               1, 16 * WIDTH).double().cpu().numpy()
    for r in range(3):
        kk, vv = (np.concatenate(x) for x in w.host[r * LAYERS + 1])
        ref = prompt.chunk_attention_request(q[r:r + 1].double().numpy(), kk, vv, w.len[r], D ** -0.5)
        assert np.abs(got[r:r + 1] - ref).max() <= 0.05


def test_without_the_marshalling_module(device, monkeypatch):
    """The same steps through ctypes, with numpy integers among the arguments."""
    monkeypatch.setattr(nsd, "_native_module", nsd._NoBinding())
    w = Worker(device, 3)
    w.step(np.array([50, 1, 0]))
    w.step(np.array([1, 1, 100]))
    nsd.trim_blocks(w.table, w.owned, w.lens, w.free, w.count, new_owned=w.owned,
                    new_free_count=w.count)
    w.step([1, 1, 1], softcap=10.0)


def test_a_pool_that_runs_short(device):
    w = Worker(device, 3)
    w.step([500, 300, 100])                       # 32 + 19 + 7 of 64 blocks
    w.step([1, 200, 40], granted=[1, 0, 0])       # 13 more do not fit, nor what comes after
    nsd.trim_blocks(w.table, w.owned, i32([0, 300, 100], device), w.free, w.count,
                    new_owned=w.owned, new_free_count=w.count)
    assert w.owned.tolist() == [0, 19, 7]
    w.lens[0] = 0
    w.len[0] = 0
    for layer in range(LAYERS):
        w.host[layer] = [[], []]
    w.step([40, 200, 41])
    w.step([1, 1, 1])


def test_a_captured_step(device):
    """Single-token steps replayed from a graph continue from one another."""
    w = Worker(device, 4)
    w.step([20, 5, 33, 64])
    rows = [tuple(t.to(device) for t in r) for r in w.rows(4)]
    indptr, pos = i32([0, 1, 2, 3, 4], device), i32([20, 5, 33, 64], device)
    freq = w.freq.to(device)
    out = torch.empty((LAYERS, 4, HQ, D), dtype=torch.bfloat16, device=device)
    ws = nsd.new_workspace(nsd.chunk_attention_workspace_size(4, 4, HQ, HKV, D, 1, 16 * WIDTH), device)
    state = [w.k, w.v, w.table, w.owned, w.lens, w.count, pos]
    start = [t.clone() for t in state]

    def step():
        prefill_chunk(w.k, w.v, rows, pos, freq, w.table, w.owned, w.lens, indptr, w.free, w.count,
                      4, 1, 16 * WIDTH, out=out, workspace=ws)
        pos.add_(1)

    eager = []
    for _ in range(20):
        step()
        eager.append(out.clone())
    for t, s in zip(state, start):
        t.copy_(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for t, s in zip(state, start):
        t.copy_(s)
    for i in range(20):
        out.fill_(3.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager[i]), i
        torch.randn(4096, device=device).sum().item()


def test_layers_of_a_model(device):
    """rows may be a function of the layer and the previous layer's output."""
    w = Worker(device, 2)
    seen = []

    def rows(layer, prev):
        seen.append((layer, None if prev is None else tuple(prev.shape)))
        base = torch.randn((7, HQ, D), generator=w.gen).bfloat16().to(device)
        q = base if prev is None else base + prev
        return q, q[:, :HKV], q[:, -HKV:]

    outs, granted, _ = prefill_chunk(w.k, w.v, rows, i32(range(7), device), w.freq.to(device), w.table,
                                     w.owned, w.lens, i32([0, 3, 7], device), w.free, w.count, 7, 4,
                                     64)
    assert seen == [(0, None), (1, (7, HQ, D))] and len(outs) == 2
    assert all(torch.isfinite(o).all() for o in outs) and granted.tolist() == [1, 1]
