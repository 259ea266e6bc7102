"""The prompt path's calls name bad arguments before anything reaches the GPU (no GPU needed)."""
import ctypes

import pytest
import torch

import paper_2609_29364_amd as nsd


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(nsd.LIB_PATH):
        from paper_2609_29364_amd.build import build
        build()
    return nsd.lib()


FAKE = 1 << 20      # never dereferenced: the checks fail first


def call(f, defaults, **kw):
    assert set(kw) <= {k for k, _ in defaults}
    return f(*[kw.get(k, v) for k, v in defaults])


PLAN = [("table", FAKE), ("width", 8), ("owned", FAKE), ("lens", FAKE), ("indptr", FAKE),
        ("bs", 4), ("total", 9), ("free", FAKE), ("capacity", 10), ("count", FAKE),
        ("new_owned", FAKE), ("new_lens", FAKE), ("new_count", FAKE), ("granted", FAKE),
        ("slots", FAKE), ("stream", None)]
TRIM = [("table", FAKE), ("width", 8), ("owned", FAKE), ("keep", FAKE), ("bs", 4), ("free", FAKE),
        ("capacity", 10), ("count", FAKE), ("new_owned", FAKE), ("new_count", FAKE),
        ("stream", None)]


@pytest.mark.parametrize("bad, status", [
    (dict(bs=-1), 2), (dict(bs=8193), 2), (dict(width=0), 2), (dict(capacity=-1), 2),
    (dict(capacity=2**27 + 1), 3), (dict(count=None), 1), (dict(table=None), 1),
    (dict(owned=None), 1), (dict(free=None), 1), (dict(new_count=None), 1)])
def test_block_calls(lib, bad, status):
    assert call(lib.nsd_plan_blocks, PLAN, **bad) == status
    assert b"plan_blocks" in lib.nsd_last_error()
    assert call(lib.nsd_trim_blocks, TRIM, **bad) == status
    assert b"trim_blocks" in lib.nsd_last_error()


def test_plan_and_trim_alone(lib):
    assert call(lib.nsd_plan_blocks, PLAN, total=-1) == 2
    for p in ("slots", "lens", "indptr", "granted", "new_lens"):
        assert call(lib.nsd_plan_blocks, PLAN, **{p: None}) == 1
    assert call(lib.nsd_trim_blocks, TRIM, keep=None) == 1
    # tables of more ids than an int32 counts
    assert call(lib.nsd_trim_blocks, TRIM, bs=8192, width=2**20) == 3


ROPE = [("k_pool", FAKE), ("v_pool", FAKE), ("nb", 100), ("q", FAKE), ("qs", 4 * 64), ("k", FAKE),
        ("ks", 2 * 64), ("v", FAKE), ("vs", 2 * 64), ("pos", FAKE), ("freq", FAKE),
        ("sections", None), ("axes", 1), ("rot", 64), ("adj", 0), ("slots", FAKE), ("total", 7),
        ("hq", 4), ("hkv", 2), ("block", 16), ("d", 64), ("out", FAKE + 16), ("stream", None)]


@pytest.mark.parametrize("bad, status", [
    (dict(block=32), 3), (dict(d=96), 3), (dict(hq=5), 2), (dict(hkv=0), 2), (dict(total=-1), 2),
    (dict(nb=-1), 2), (dict(nb=2**27 + 1), 3), (dict(nb=2**27, hkv=16, hq=16), 3),
    (dict(rot=24), 2), (dict(rot=80), 2), (dict(rot=-16), 2), (dict(axes=0), 2), (dict(axes=5), 2),
    (dict(axes=2), 1), (dict(q=None), 1), (dict(k=None), 1), (dict(v=None), 1), (dict(pos=None), 1),
    (dict(freq=None), 1), (dict(slots=None), 1), (dict(out=None), 1), (dict(k_pool=None), 1),
    (dict(qs=4 * 64 - 8), 2), (dict(ks=64), 2), (dict(vs=2 * 64 + 4), 2), (dict(q=FAKE + 8), 2),
    (dict(out=FAKE + 4), 2), (dict(v_pool=FAKE + 2), 2), (dict(out=FAKE, qs=4 * 64 + 8), 2)])
def test_rope_append(lib, bad, status):
    assert call(lib.nsd_rope_append, ROPE, **bad) == status
    assert b"rope_append" in lib.nsd_last_error()


def test_rope_sections(lib):
    for cuts, status in (((16, 8), 2), ((40, -8), 2), ((33, 0), 2), ((2**31 - 1, 33), 2)):
        a = (ctypes.c_int32 * 2)(*cuts)
        assert call(lib.nsd_rope_append, ROPE, axes=2, sections=a) == status
    a = (ctypes.c_int32 * 2)(16, 16)
    assert call(lib.nsd_rope_append, ROPE, axes=2, sections=a, total=0) == 0
    assert call(lib.nsd_rope_append, ROPE, total=0) == 0


CHUNK = [("q", FAKE), ("k", FAKE), ("v", FAKE), ("nb", 64), ("bt", FAKE), ("width", 16),
         ("sl", FAKE), ("qi", FAKE), ("bs", 4), ("total", 30), ("hq", 4), ("hkv", 2), ("d", 64),
         ("blk", 16), ("mq", 20), ("msl", 256), ("scale", 0.125), ("cap", 0.0), ("slopes", None),
         ("first", None), ("prefix", None), ("out", FAKE), ("ws", None), ("wsb", 0),
         ("stream", None)]


@pytest.mark.parametrize("bad, status", [
    (dict(bs=-1), 2), (dict(bs=8193), 2), (dict(blk=32), 3), (dict(d=80), 3), (dict(hq=5), 2),
    (dict(hkv=0), 2), (dict(total=-1), 2), (dict(mq=0), 2), (dict(msl=0), 2), (dict(width=0), 2),
    (dict(nb=-1), 2), (dict(nb=2**31), 3), (dict(nb=2**30, hkv=4, hq=4), 3),
    (dict(total=2**30), 3), (dict(scale=float("nan")), 2), (dict(scale=float("inf")), 2),
    (dict(cap=-1.0), 2), (dict(cap=float("nan")), 2), (dict(cap=float("inf")), 2),
    (dict(q=None), 1), (dict(k=None), 1), (dict(v=None), 1), (dict(bt=None), 1), (dict(sl=None), 1),
    (dict(qi=None), 1), (dict(out=None), 1), (dict(q=FAKE + 2), 2), (dict(v=FAKE + 8), 2)])
def test_chunk_attention(lib, bad, status):
    assert call(lib.nsd_chunk_attention, CHUNK, **bad) == status
    assert b"chunk_attention" in lib.nsd_last_error()


def test_chunk_attention_workspace(lib):
    size = lib.nsd_chunk_attention_workspace_size
    assert size(1, 1, 32, 8, 128, 1, 32768) > 0           # one long request is split
    assert size(256, 256, 32, 8, 128, 1, 4096) == 0       # a full device is not
    assert size(4, 30, 5, 2, 64, 20, 256) == 0            # invalid sizes
    assert size(8193, 30, 4, 2, 64, 20, 256) == 0
    need = size(1, 1, 32, 8, 128, 1, 32768)
    args = dict(bs=1, total=1, hq=32, hkv=8, d=128, mq=1, msl=32768, width=2048)
    assert call(lib.nsd_chunk_attention, CHUNK, **args) == 4
    assert call(lib.nsd_chunk_attention, CHUNK, ws=FAKE, wsb=need - 1, **args) == 4
    assert call(lib.nsd_chunk_attention, CHUNK, ws=FAKE + 4, wsb=need, **args) == 4
    assert b"workspace" in lib.nsd_last_error()
    assert call(lib.nsd_chunk_attention, CHUNK, bs=0) == 0
    assert call(lib.nsd_chunk_attention, CHUNK, total=0) == 0


def test_the_binding_names_tensors_off_the_gpu():
    i = torch.zeros(4, dtype=torch.int32)
    b = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="block_table must be on a GPU"):
        nsd.plan_blocks(i.view(2, 2), i, i, i, i, i, 4)
    with pytest.raises(ValueError, match="block_table must be on a GPU"):
        nsd.trim_blocks(i.view(2, 2), i, i, i, i)
    with pytest.raises(ValueError, match="q must be on a GPU"):
        nsd.rope_append(b, b, b, b, b, i, i, i)
    with pytest.raises(ValueError, match="q must be on a GPU"):
        nsd.chunk_attention(b, b, b, i, i, i, 1, 1)
    with pytest.raises(TypeError, match="q must be torch.bfloat16"):
        nsd.chunk_attention(b.float(), b, b, i, i, i, 1, 1)
