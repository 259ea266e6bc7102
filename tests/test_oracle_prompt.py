"""Pins of the prompt path's oracle: conservation of blocks, rotations, and attention against the
verification oracle and a dense masked softmax."""
import numpy as np
import pytest
import torch

import oracle
from oracle import prompt


def test_plan_takes_from_the_top_and_trim_gives_back():
    table = np.full((3, 4), -1, np.int32)
    table[0, 0], table[2, :2] = 9, (7, 8)
    free = np.array([3, 1, 5, 2, 4], np.int32)
    t, owned, lens, left, granted, slots = prompt.plan_blocks(
        table, [1, 0, 2], [15, 0, 32], [0, 2, 2, 35], free, 5, 35)
    # request 0: one more token in block 9, one in the first free block
    assert t[0, :2].tolist() == [9, 4] and slots[:2].tolist() == [9 * 16 + 15, 4 * 16]
    # request 1 has no token; request 2 needs 3 blocks more than its row holds
    assert granted.tolist() == [1, 1, 0] and owned.tolist() == [2, 0, 2] and left == 4
    assert lens.tolist() == [17, 0, 32] and (slots[2:] == -1).all()
    owned, free, left = prompt.trim_blocks(t, owned, [16, 0, 0], free, left)
    # block 4 goes back on top; of request 2's blocks the list holds no more
    assert owned.tolist() == [1, 0, 0] and left == 5 and free.tolist() == [3, 1, 5, 2, 4]


def test_plan_serves_a_prefix_when_blocks_run_short():
    table = np.full((4, 8), -1, np.int32)
    _, owned, _, left, granted, _ = prompt.plan_blocks(
        table, [0, 0, 0, 0], [0, 0, 0, 0], [0, 32, 112, 112, 113], np.arange(4), 4, 113)
    assert granted.tolist() == [1, 0, 1, 0] and owned.tolist() == [2, 0, 0, 0] and left == 2


def test_blocks_are_conserved():
    rng = np.random.default_rng(0)
    bs, width, pool = 9, 12, 60
    table = np.full((bs, width), -1, np.int64)
    owned, lens = np.zeros(bs, int), np.zeros(bs, int)
    free, left = rng.permutation(pool), pool
    for _ in range(40):
        n = rng.integers(0, 40, bs)
        indptr = np.concatenate([[0], np.cumsum(n)])
        table, owned, lens, left, granted, slots = prompt.plan_blocks(
            table, owned, lens, indptr, free, left, indptr[-1])
        used = slots[slots >= 0]
        assert len(set(used.tolist())) == len(used)
        lens = np.minimum(lens, rng.integers(0, 16 * width, bs))
        owned, free, left = prompt.trim_blocks(table, owned, lens, free, left)
        ids = [int(x) for r in range(bs) for x in table[r, :owned[r]]] + free[:left].tolist()
        assert sorted(ids) == list(range(pool))


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_depends_on_relative_positions(interleaved):
    rng = np.random.default_rng(1)
    q, k = rng.standard_normal((2, 1, 1, 64))
    freq = 1e4 ** (-np.arange(24) / 24)
    dots = []
    for shift in (0, 5, 1000):
        a = prompt.rotate(q, [[7 + shift]], freq, None, interleaved)
        b = prompt.rotate(k, [[3 + shift]], freq, None, interleaved)
        assert np.allclose(np.linalg.norm(a), np.linalg.norm(q))
        assert np.array_equal(a[..., 48:], q[..., 48:])
        dots.append(float((a * b).sum()))
    assert np.allclose(dots, dots[0])
    # complex multiplication, axis by axis
    pos = np.array([[2], [3], [5]])
    got = prompt.rotate(q, pos, freq, [10, 6, 8], interleaved)
    x = q[0, 0, 0:48:2] + 1j * q[0, 0, 1:48:2] if interleaved else q[0, 0, :24] + 1j * q[0, 0, 24:48]
    z = x * np.exp(1j * np.repeat([2, 3, 5], [10, 6, 8]) * freq)
    ref = np.stack([z.real, z.imag], -1).reshape(-1) if interleaved else np.concatenate([z.real, z.imag])
    assert np.allclose(got[0, 0, :48], ref)


def test_chunk_attention_is_verification_without_options():
    rng = np.random.default_rng(2)
    q, k, v = (rng.standard_normal(s) for s in ((5, 4, 8), (19, 2, 8), (19, 2, 8)))
    assert np.allclose(prompt.chunk_attention_request(q, k, v, 19, 0.3),
                       oracle.attention.verify_attention_request(q, k, v, 0.3))


def test_chunk_attention_against_a_dense_masked_softmax():
    rng = np.random.default_rng(3)
    n, length, prefix, cap = 7, 30, 9, 3.0
    q, k, v = (rng.standard_normal(s) for s in ((n, 4, 8), (length, 2, 8), (length, 2, 8)))
    first = np.array([0, 12, 24, 29, 20, 27, 40])
    slopes = np.array([0.0, 0.1, 0.5, 2.0])
    valid = np.ones(length, bool)
    valid[3:5] = False
    got = prompt.chunk_attention_request(q, k, v, length, 0.7, cap, slopes, first, prefix, valid)
    p, t = np.arange(length - n, length)[:, None], np.arange(length)[None, :]
    see = ((t < prefix) | ((t <= p) & (t >= first[:, None]))) & valid
    x = torch.from_numpy(cap * np.tanh(0.7 * np.einsum("nhd,thd->hnt", q, k.repeat(2, 1)) / cap)
                         - slopes[:, None, None] * np.abs(p - t))
    w = x.masked_fill(~torch.from_numpy(see), -torch.inf).softmax(-1).numpy()
    assert np.allclose(got, np.einsum("hnt,thd->nhd", w, v.repeat(2, 1)))


def test_rows_that_see_nothing_are_zero():
    q, k, v = np.ones((3, 1, 4)), np.full((5, 1, 4), np.nan), np.full((5, 1, 4), np.inf)
    first = np.array([9, 9, 9])
    assert (prompt.chunk_attention_request(q, k, v, 5, 1.0, first_keys=first) == 0).all()
    # more queries than tokens: the rows before position 0 see nothing
    out = prompt.chunk_attention_request(q, np.ones((2, 1, 4)), np.ones((2, 1, 4)), 2, 1.0)
    assert (out[0] == 0).all() and (out[1:] == 1).all()
