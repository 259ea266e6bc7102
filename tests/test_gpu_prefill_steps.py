"""prefill_chunk against the calls that it composes: the same bits, and padded to a fixed number of
rows as a captured step is."""
import numpy as np
import pytest
import torch

import paper_2609_29364_amd as nsd
from paper_2609_29364_amd.round import prefill_chunk
from parity import i32

pytestmark = pytest.mark.gpu

LAYERS, POOL, WIDTH = 2, 60, 40


class State:
    def __init__(self, dev, bs, hkv, d, seed=0):
        rng = np.random.default_rng(seed)
        z = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device=dev)
        self.k, self.v = z(LAYERS, POOL, hkv, d // 8, 16, 8), z(LAYERS, POOL, hkv, d, 16)
        self.table = i32(np.full((bs, WIDTH), -1), dev)
        self.owned, self.lens = i32([0] * bs, dev), i32([0] * bs, dev)
        self.free, self.count = i32(rng.permutation(POOL), dev), i32([POOL], dev)

    def all(self):
        return [self.k, self.v, self.table, self.owned, self.lens, self.free, self.count]


@pytest.mark.parametrize("pad", [0, 1, 300])
@pytest.mark.parametrize("hq, hkv, d, options", [
    (8, 2, 64, {}), (4, 4, 128, dict(softcap=30.0)), (6, 1, 64, dict(window=50, prefix=7))])
def test_a_step_is_its_calls(device, hq, hkv, d, options, pad):
    bs, dev = 3, device
    g = torch.Generator().manual_seed(pad + d)
    a, b = State(dev, bs, hkv, d), State(dev, bs, hkv, d)
    freq = torch.tensor(1e4 ** (-np.arange(d // 2) / (d // 2)), dtype=torch.float32, device=dev)
    ctx = np.zeros(bs, int)
    # the last step's second request asks for more blocks than are left, the others for none
    for new in ([50, 1, 0], [130, 70, 1], [1, 1, 300], [1, 500, 1]):
        indptr = np.concatenate([[0], np.cumsum(new)])
        n, total = int(indptr[-1]), int(indptr[-1]) + pad
        pos = np.concatenate([np.arange(c, c + m) for c, m in zip(ctx, new)] + [np.full(pad, 5)])
        rows = [tuple(torch.randn((total, h, d), generator=g).bfloat16().to(dev)
                      for h in (hq, hkv, hkv)) for _ in range(LAYERS)]
        kw = {k: x for k, x in options.items() if k == "softcap"}
        if "window" in options:
            kw.update(first_keys=i32(np.maximum(pos - options["window"], 0), dev),
                      prefix_lens=i32([options["prefix"]] * bs, dev))
        out = torch.full((LAYERS, total, hq, d), 7.0, dtype=torch.bfloat16, device=dev)
        _, granted, slots = prefill_chunk(a.k, a.v, rows, i32(pos, dev), freq, a.table, a.owned,
                                          a.lens, i32(indptr, dev), a.free, a.count, total,
                                          max(new), 16 * WIDTH, out=out, **kw)
        # the same without the padding
        b.owned, b.lens, b.count, gr, sl = nsd.plan_blocks(b.table, b.owned, b.lens,
                                                           i32(indptr, dev), b.free, b.count, n)
        assert torch.equal(gr, granted) and torch.equal(sl, slots[:n]) and (slots[n:] == -1).all()
        if "first_keys" in kw:
            kw["first_keys"] = kw["first_keys"][:n]
        for layer, (q, k, v) in enumerate(rows):
            q = nsd.rope_append(b.k[layer], b.v[layer], q[:n], k[:n], v[:n], i32(pos[:n], dev), freq,
                                sl)
            o = nsd.chunk_attention(q, b.k[layer], b.v[layer], b.table, b.lens, i32(indptr, dev),
                                    max(new), 16 * WIDTH, **kw)
            # Padding can change the items' size, and with it what weights are rounded against: twice
            # half a step of every weight and of the output.
            tol = 0 if pad == 0 else 4 * 2.0**-8 * v.abs().max().item()
            assert (out[layer, :n].float() - o.float()).abs().max() <= tol
            assert (out[layer, n:] == 7).all()
        for x, y in zip(a.all(), b.all()):
            assert torch.equal(x, y)
        ctx = a.lens.cpu().numpy().astype(int)
    assert granted.tolist() == [1, 0, 1]
