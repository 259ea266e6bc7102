"""Rotary rows into the cache against the oracle.

An output is within half a bf16 step of a value computed in fp32: 2^-8 of the value, plus, with
|x| + |y| the pair's size, 1e-6 (|x| + |y|): the angle's error (half a step of a turn's fraction
in fp32, 2^-25 turns = 1.9e-7), the sine's and cosine's (2 steps, 2.4e-7) and the two products and
their sum (1.8e-7).  Values and dimensions that pass are equal."""
import numpy as np
import pytest
import torch

import paper_2609_29364_amd as nsd
from oracle import prompt
from parity import i32, u16

pytestmark = pytest.mark.gpu


def make(dev, seed, n, hq, hkv, d, rot, axes=1, blocks=40, fused=True, far=40000):
    g = torch.Generator().manual_seed(seed)
    rng = np.random.default_rng(seed)
    rows = torch.randn((n, (hq + 2 * hkv) * d + (8 if fused else 0)), generator=g).bfloat16()
    rows = rows.to(dev)
    cut = [hq * d, (hq + hkv) * d, (hq + 2 * hkv) * d]
    q, k, v = (rows[:, a:b].view(n, h, d) for a, b, h in
               ((0, cut[0], hq), (cut[0], cut[1], hkv), (cut[1], cut[2], hkv)))
    if not fused:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    pairs = rot // 2
    sections = None
    if axes > 1:
        cuts = np.sort(rng.integers(0, pairs + 1, axes - 1))
        sections = np.diff(np.concatenate([[0], cuts, [pairs]])).tolist()
    pos = rng.integers(-3, far, (axes, n)).astype(np.int32)
    freq = (1e6 ** (-np.arange(pairs) / max(1, pairs))).astype(np.float32)
    planes = [torch.randn(s, generator=g).bfloat16().to(dev)
              for s in ((blocks, hkv, d // 8, 16, 8), (blocks, hkv, d, 16))]
    return q, k, v, pos, freq, sections, planes


def near(got, x, ref, interleaved, pairs):
    """|got - ref| within the bound of the module's text; x: the rows before turning."""
    size = np.zeros_like(ref)
    a = np.abs(x)
    if interleaved:
        both = a[..., 0:2 * pairs:2] + a[..., 1:2 * pairs:2]
        size[..., 0:2 * pairs:2] = size[..., 1:2 * pairs:2] = both
    else:
        both = a[..., :pairs] + a[..., pairs:2 * pairs]
        size[..., :pairs] = size[..., pairs:2 * pairs] = both
    err = np.abs(got - ref)
    assert np.isfinite(got).all()
    assert (err <= 2.0**-8 * np.abs(ref) + 1e-6 * size).all(), float(err.max())


def host(t):
    return t.double().cpu().numpy()


def check(dev, n, hq, hkv, d, rot, slots, axes=1, interleaved=False, fused=True, blocks=40,
          in_place=False, far=40000):
    q, k, v, pos, freq, sections, (kp, vp) = make(dev, n + rot, n, hq, hkv, d, rot, axes, blocks,
                                                  fused, far)
    before = [u16(x).copy() for x in (kp, vp)]
    q0, k0, v0 = host(q), host(k), u16(v).copy()
    out = nsd.rope_append(kp, vp, q, k, v, i32(pos if axes > 1 else pos[0], dev),
                          torch.from_numpy(freq).to(dev), i32(slots, dev), sections=sections,
                          interleaved=interleaved, q_out=q if in_place else None)
    assert out is q or not in_place
    near(host(out), q0, prompt.rotate(q0, pos, freq, sections, interleaved), interleaved, rot // 2)
    kref = prompt.rotate(k0, pos, freq, sections, interleaved)
    kt, vt = kp.transpose(2, 3).reshape(blocks, hkv, 16, d), vp.transpose(2, 3)   # [block][head][slot][D]
    rows = np.flatnonzero((slots >= 0) & (slots < 16 * blocks))
    b, s = slots[rows] // 16, slots[rows] % 16
    near(host(kt)[b, :, s], k0[rows], kref[rows], interleaved, rot // 2)
    assert np.array_equal(u16(vt.contiguous())[b, :, s], v0[rows])
    if rot < d:
        assert np.array_equal(host(kt)[b, :, s][..., rot:], k0[rows][..., rot:])
    # every other slot is as it was
    hit = np.zeros((blocks, 16), bool)
    hit[b, s] = True
    for now, old, axis in ((u16(kp), before[0], 3), (u16(vp), before[1], 3)):
        now, old = (np.moveaxis(x, axis, 1).reshape(blocks, 16, -1) for x in (now, old))
        assert np.array_equal(now[~hit], old[~hit])


def runs(lengths, starts):
    """Slots of requests of these lengths, each beginning at its start in its own blocks."""
    out, block = [], 0
    for n, s in zip(lengths, starts):
        t = np.arange(s, s + n)
        ids = np.array([(7 * (block + i)) % 37 for i in range(t[-1] // 16 + 1)]) if n else t
        block += t[-1] // 16 + 1 if n else 0
        out.append(ids[t // 16] * 16 + t % 16)
    return np.concatenate(out)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("hq, hkv, d, rot", [(4, 2, 64, 64), (8, 8, 128, 128), (7, 1, 128, 64),
                                             (6, 2, 64, 16), (32, 8, 128, 128), (2, 2, 128, 0)])
def test_heads_and_widths(device, hq, hkv, d, rot, interleaved):
    check(device, 53, hq, hkv, d, rot, runs((1, 30, 5, 17), (15, 3, 0, 16)),
          interleaved=interleaved)


@pytest.mark.parametrize("axes", [2, 3, 4])
@pytest.mark.parametrize("fused", [False, True])
def test_axes(device, axes, fused):
    check(device, 40, 8, 2, 128, 128, runs((40,), (9,)), axes=axes, fused=fused)


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 100, 500])
def test_lengths(device, n):
    start = n % 16
    check(device, n, 4, 2, 64, 64, runs((n,), (start,)), blocks=40)


def test_single_tokens(device):
    slots = np.arange(300) * 16 + np.arange(300) * 5 % 16
    check(device, 300, 16, 8, 128, 128, slots, blocks=300)


def test_slots_in_any_order(device):
    rng = np.random.default_rng(0)
    check(device, 400, 4, 2, 64, 64, rng.permutation(640)[:400])
    check(device, 320, 4, 2, 64, 64, np.arange(320)[::-1].copy())
    # neighbours in one block's order whose blocks differ, and runs that begin inside a block
    check(device, 64, 4, 2, 64, 32, np.concatenate([np.arange(7, 23), np.arange(40, 71),
                                                    np.arange(100, 117)]))


def test_rows_without_a_slot_are_turned_only(device):
    slots = runs((60,), (4,))
    slots[[0, 1, 17, 30, 59]] = [-1, -2**31, 16 * 40, 2**31 - 1, 16 * 40 + 5]
    check(device, 60, 4, 2, 64, 64, slots)


def test_in_place(device):
    check(device, 70, 8, 2, 128, 128, runs((70,), (1,)), fused=False, in_place=True)
    q, k, v, pos, freq, _, (kp, vp) = make(device, 1, 9, 4, 2, 64, 64)
    with pytest.raises(nsd.NsdError, match="dense"):       # a strided q has no room for its result
        nsd.lib()
        nsd._check("rope_append", nsd.lib().nsd_rope_append(
            kp.data_ptr(), vp.data_ptr(), 40, q.data_ptr(), q.stride(0), k.data_ptr(), k.stride(0),
            v.data_ptr(), v.stride(0), 16, 16, None, 1, 64, 0, 16, 9, 4, 2, 16, 64, q.data_ptr(),
            None))


def test_far_positions(device):
    check(device, 50, 2, 1, 64, 64, runs((50,), (0,)), far=2**31 - 1)


def test_nothing_to_do(device):
    q, k, v, pos, freq, _, (kp, vp) = make(device, 1, 0, 4, 2, 64, 64, fused=False)
    e = torch.empty(0, dtype=torch.int32, device=device)
    out = nsd.rope_append(kp, vp, q, k, v, e, torch.ones(32, device=device), e)
    assert out.shape == (0, 4, 64)


def test_refusals(device):
    q, k, v, pos, freq, _, (kp, vp) = make(device, 1, 9, 4, 2, 64, 64)
    pos, freq, s = i32(pos[0], device), torch.from_numpy(freq).to(device), i32(range(9), device)
    ok = lambda **kw: nsd.rope_append(*[kw.get(n, x) for n, x in dict(
        kp=kp, vp=vp, q=q, k=k, v=v, pos=pos, freq=freq, s=s).items()])
    ok()
    for bad in (dict(k=k[:8]), dict(vp=vp[:, :1]), dict(pos=pos[:8]), dict(s=s[:5]),
                dict(q=q.transpose(0, 1)), dict(pos=pos.view(1, 9).expand(2, 9).contiguous())):
        with pytest.raises(ValueError):
            ok(**bad)
    for bad in (dict(pos=pos.long()), dict(freq=freq.double()), dict(q=q.float())):
        with pytest.raises(TypeError):
            ok(**bad)
    with pytest.raises(nsd.NsdError, match="rot_dim"):
        ok(freq=torch.ones(33, device=device))
    with pytest.raises(nsd.NsdError, match="sections"):
        nsd.rope_append(kp, vp, q, k, v, pos.view(1, 9).repeat(2, 1), freq, s, sections=[30, 1])
    with pytest.raises(nsd.NsdError, match="aligned"):
        ok(q=torch.zeros((9, 4 * 64 + 4), dtype=torch.bfloat16, device=device)[:, 4:].view(9, 4, 64))
