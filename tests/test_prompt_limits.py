"""Limits of the prompt path's calls that no allocation reaches, refused on the host (no GPU)."""
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
