"""Argument checks of the calls on several new tokens per sequence: no CUDA call is made on these paths, and the fake pointers are never read."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def rkv():
    from paper_2505_24133_b200 import build as b
    b.build()
    import paper_2505_24133_b200 as r
    return r


def _desc(rkv, **kw):
    d = rkv.rkv_desc_default()
    d.batch, d.n_kv_heads, d.n_q_heads = 2, 8, 32
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def _tokens(rkv, **kw):
    t = rkv.rkv_tokens(20, 16)
    t.offsets = 0x30000
    for k, v in kw.items():
        setattr(t, k, v)
    return t


GOOD = 0x20000


@pytest.mark.parametrize("case,want", [
    (dict(k_cache=None), 1), (dict(v_new=None), 1), (dict(seq=None), 1), (dict(k_new=GOOD + 8), 1), (dict(q_out=GOOD + 2), 1),
    (dict(q_out=None), 1), (dict(q_new=None), 1), (dict(seq=GOOD + 2), 1), (dict(budget=0), 1), (dict(buffer=-1), 1),
    (dict(budget=1 << 20, buffer=1), 2), (dict(desc=dict(head_dim=96)), 2), (dict(desc=dict(dtype=7)), 2), (dict(desc=dict(n_q_heads=30)), 1),
    (dict(desc=dict(batch=0)), 1), (dict(desc=dict(block_table=GOOD, pool_pages=0), budget=128, buffer=0), 1),
    (dict(desc=dict(block_table=GOOD, pool_pages=9), budget=100, buffer=1), 1), (dict(desc=dict(block_table=GOOD + 1, pool_pages=9), budget=128, buffer=0), 1),
    (dict(tokens=dict(total=-1)), 1), (dict(tokens=dict(longest=0)), 1), (dict(tokens=dict(offsets=0x30001)), 1),
    (dict(tokens=dict(offsets=None)), 1), (dict(tokens=dict(total=1 << 27)), 2),
    (dict(tokens=dict(k_stride=1023)), 1), (dict(tokens=dict(k_stride=1028)), 1), (dict(tokens=dict(q_stride=4095)), 1),
    (dict(tokens=dict(out_stride=-4096)), 1), (dict(tokens=dict(v_stride=1 << 62)), 1),
    (dict(rotary=dict(dim=8)), 1), (dict(rotary=dict(dim=144)), 1), (dict(rotary=dict(dim=-16)), 1), (dict(rotary=dict(table=None)), 1),
    (dict(rotary=dict(table=GOOD + 4)), 1), (dict(rotary=dict(rows=0)), 1), (dict(rotary=dict(positions=GOOD + 1)), 1),
    (dict(q_new=GOOD, q_out=GOOD, tokens=dict(q_stride=8192)), 1),
    (dict(tokens=dict(total=0)), 0), (dict(tokens=dict(total=0), q_new=None, q_out=None), 0),
])
def test_append_rotary_refuses(rkv, case, want):
    a = dict(k_cache=GOOD, v_cache=GOOD, k_new=GOOD, v_new=GOOD, seq=GOOD, q_new=GOOD, q_out=2 * GOOD, budget=1024, buffer=128)
    a.update({k: v for k, v in case.items() if k in a})
    rotary = rkv.rkv_rotary(None, 128)
    rotary.table, rotary.rows = GOOD, 100
    for k, v in case.get("rotary", {}).items():
        setattr(rotary, k, v)
    got = rkv.rkv_append_rotary(_desc(rkv, **case.get("desc", {})), a["k_cache"], a["v_cache"], a["k_new"], a["v_new"], a["seq"], a["budget"],
                                a["buffer"], _tokens(rkv, **case.get("tokens", {})), rotary, a["q_new"], a["q_out"], 0)
    assert got == want


def test_structures_are_taken_as_what_they_are(rkv):
    d, t, r = _desc(rkv), _tokens(rkv), rkv.rkv_rotary(None, 0)
    call = lambda d, t, r: rkv.rkv_append_rotary(d, None, None, None, None, None, 64, 32, t, r, None, None, 0)  # noqa: E731
    assert call(d, t, r) == 1                                     # null tensors
    for bad in ((t, t, r), (d, t, t), (d, t, d)):
        with pytest.raises(TypeError):
            call(*bad)
    for bad in (b"0" * 64, None, (ctypes.c_char * 64)()):
        with pytest.raises(TypeError):
            call(bad, t, r)
        with pytest.raises(TypeError):
            call(d, t, bad)


def test_token_tensors_have_the_strides_they_are_said_to_have(rkv):
    d, r = _desc(rkv, n_kv_heads=2, n_q_heads=2, head_dim=64), rkv.rkv_rotary(None, 0)
    qkv = torch.zeros(4, 6, 64, dtype=torch.bfloat16)
    t = rkv.rkv_tokens(4, 4, k_stride=384, v_stride=384)
    with pytest.raises(AssertionError):
        rkv.rkv_append_rotary(d, None, None, qkv[:, :2].contiguous(), qkv[:, 2:4], None, 64, 32, t, r, None, None, 0)
    with pytest.raises(AssertionError):
        rkv.rkv_append_rotary(d, None, None, qkv[:, 0:4:2], qkv[:, 2:4], None, 64, 32, t, r, None, None, 0)
    with pytest.raises(AssertionError):                           # strided, but the call was not told
        rkv.rkv_append_rotary(d, None, None, qkv[:, :2], qkv[:, 2:4], None, 64, 32, rkv.rkv_tokens(4, 4), r, None, None, 0)
    assert rkv.rkv_append_rotary(d, None, None, qkv[:, :2], qkv[:, 2:4], None, 64, 32, t, r, None, None, 0) == 1


@pytest.mark.parametrize("case,want", [
    (dict(k_cache=None), 1), (dict(q=None), 1), (dict(out=None), 1), (dict(seq=None), 1), (dict(q=GOOD + 8), 1), (dict(out=GOOD + 4), 1),
    (dict(seq=GOOD + 2), 1), (dict(window=-1), 1), (dict(sinks=-1), 1), (dict(budget=0), 1), (dict(budget=1 << 20), 2),
    (dict(desc=dict(head_dim=96)), 2), (dict(desc=dict(n_q_heads=30)), 1), (dict(tokens=dict(q_stride=4100)), 1),
    (dict(tokens=dict(out_stride=4095)), 1), (dict(tokens=dict(longest=0)), 1), (dict(tokens=dict(offsets=None)), 1),
    (dict(desc=dict(block_table=GOOD, pool_pages=9)), 1), (dict(desc=dict(workspace=None)), 3), (dict(desc=dict(workspace=0x10010)), 3),
    (dict(desc=dict(workspace_bytes=1024)), 3), (dict(tokens=dict(total=0)), 0),
])
def test_window_attention_refuses(rkv, case, want):
    a = dict(k_cache=GOOD, v_cache=GOOD, q=GOOD, seq=GOOD, out=GOOD, budget=1000, buffer=1, window=100, sinks=4)
    a.update({k: v for k, v in case.items() if k in a})
    d = _desc(rkv, workspace=0x10000, workspace_bytes=1 << 40)
    for k, v in case.get("desc", {}).items():
        setattr(d, k, v)
    t = _tokens(rkv, **case.get("tokens", {}))
    assert rkv.rkv_window_attention(d, a["k_cache"], a["v_cache"], a["q"], a["seq"], a["out"], a["budget"], a["buffer"], t, a["window"],
                                    a["sinks"], 0) == want


@pytest.mark.parametrize("case,want", [
    (dict(k_cache=None), 1), (dict(q=None), 1), (dict(out=GOOD + 8), 1), (dict(seq=GOOD + 1), 1), (dict(budget=0), 1),
    (dict(prefix=dict(k=None)), 1), (dict(prefix=dict(v=GOOD + 4)), 1), (dict(prefix=dict(lens=None)), 1), (dict(prefix=dict(lens=GOOD + 2)), 1),
    (dict(prefix=dict(count=0)), 1), (dict(prefix=dict(count=3)), 1), (dict(prefix=dict(rows=0)), 1), (dict(prefix=dict(rows=(1 << 20) + 1)), 2),
    (dict(prefix=dict(table=GOOD, pages=4, rows=100)), 1), (dict(prefix=dict(table=GOOD, pages=0, rows=128)), 1),
    (dict(prefix=dict(table=GOOD + 2, pages=4, rows=128)), 1), (dict(desc=dict(workspace=None)), 3), (dict(desc=dict(workspace_bytes=256)), 3),
    (dict(desc=dict(dtype=5)), 2),
])
def test_prefix_attention_refuses(rkv, case, want):
    a = dict(k_cache=GOOD, v_cache=GOOD, q=GOOD, seq=GOOD, out=GOOD, budget=1000, buffer=1)
    a.update({k: v for k, v in case.items() if k in a})
    d = _desc(rkv, workspace=0x10000, workspace_bytes=1 << 40)
    for k, v in case.get("desc", {}).items():
        setattr(d, k, v)
    x = rkv.RkvPrefix(GOOD, GOOD, 2, 100000, GOOD, None, 0)
    for k, v in case.get("prefix", {}).items():
        setattr(x, k, v)
    assert rkv.rkv_prefix_attention(d, a["k_cache"], a["v_cache"], a["q"], a["seq"], a["out"], a["budget"], a["buffer"], x, 0) == want


def test_workspace_sizes(rkv):
    """Zero for what is refused, and of the window attention for calls that fill the GPU."""
    d, t = _desc(rkv), _tokens(rkv)
    assert rkv.rkv_window_workspace_bytes(d, 1000, 1, t, -1, 0) == 0 and rkv.rkv_window_workspace_bytes(_desc(rkv, head_dim=32), 1000, 1, t, 0, 0) == 0
    assert rkv.rkv_window_workspace_bytes(_desc(rkv, batch=512), 1000, 1, rkv.rkv_tokens(512 * 64, 64), 0, 0) == 0
    x = rkv.RkvPrefix(GOOD, GOOD, 2, 100000, GOOD, None, 0)
    assert rkv.rkv_prefix_workspace_bytes(d, 1000, 1, x) > 0 and rkv.rkv_prefix_workspace_bytes(_desc(rkv, batch=3), 1000, 1, x) == 0


@pytest.mark.parametrize("dtype,d", [("RKV_BF16", 128), ("RKV_BF16", 64), ("RKV_FP8_E4M3", 128)])
@pytest.mark.parametrize("batch,cap,window", [(16, 32768, 0), (8, 40960, 0), (9, 30848, 0), (5, 57344, 0), (8, 1 << 20, 35000)])
def test_more_shares_than_a_cluster_has_blocks_have_room(rkv, dtype, d, batch, cap, window):
    """Single tokens of many heads over so many rows that a head's keys go to more than 16 blocks, the most of a cluster: the blocks' partial
    results have a place in the workspace."""
    desc = _desc(rkv, batch=batch, dtype=getattr(rkv, dtype), head_dim=d, block_table=GOOD, pool_pages=9)
    tokens = rkv.rkv_tokens(batch, 1)
    assert rkv.rkv_window_workspace_bytes(desc, cap - 128, 128, tokens, window, 0) >= batch * 32 * 17 * (d + 4) * 4
    x = rkv.RkvPrefix(GOOD, GOOD, batch, 128, GOOD, GOOD, 9)         # a short prefix for each, read by the same blocks
    if window == 0 and cap < 57344:
        assert rkv.rkv_prefix_workspace_bytes(desc, cap - 128, 128, x) >= batch * 32 * 17 * (d + 4) * 4
