"""Limits of the prompt path's calls that no allocation reaches, refused on the host, and the bound
of its workspaces (no GPU)."""
import random

import pytest

from test_prompt_refusals import CHUNK, ROPE, call, lib  # noqa: F401


@pytest.mark.parametrize("total, heads", [(2**27, 1), (2**31 - 1, 1), (2**23, 512)])
def test_rows_past_one_launch(lib, total, heads):
    """2^24 workgroups of 256 threads are more than a launch takes."""
    assert call(lib.nsd_rope_append, ROPE, total=total, hq=heads, hkv=heads, qs=heads * 64,
                ks=heads * 64, vs=heads * 64) == 3
    assert b"rope_append" in lib.nsd_last_error() and b"workgroups" in lib.nsd_last_error()


@pytest.mark.parametrize("bs, heads", [(8192, 2048), (8192, 2**20), (5000, 4096)])
def test_items_past_one_launch(lib, bs, heads):
    assert call(lib.nsd_chunk_attention, CHUNK, bs=bs, total=1, hq=heads, hkv=heads, nb=1) == 3
    assert b"chunk_attention" in lib.nsd_last_error() and b"workgroups" in lib.nsd_last_error()


def test_one_workspace_for_every_batch(lib):
    size, bound = lib.nsd_chunk_attention_workspace_size, lib.nsd_chunk_attention_workspace_bound
    # a smaller batch can need more than a larger one
    assert size(100, 100, 32, 8, 128, 1, 4096) > size(256, 256, 32, 8, 128, 1, 4096)
    rng = random.Random(0)
    reached = set()
    for _ in range(20000):
        hkv, d = rng.choice([1, 2, 3, 8, 32, 100, 513, 1025]), rng.choice([64, 128])
        bs, total = int(2 ** rng.uniform(0, 13)), int(2 ** rng.uniform(0, 16))
        n = size(bs, total, hkv * rng.choice([1, 4, 7]), hkv, d, 1, int(2 ** rng.uniform(0, 31)) - 1)
        assert n <= bound(hkv, d)
        if n == bound(hkv, d) > 0:
            reached.add(hkv)
    assert {1, 2, 3, 8, 32, 100} <= reached
    assert bound(0, 64) == bound(8, 80) == bound(-1, 128) == bound(1025, 128) == 0
