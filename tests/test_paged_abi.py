"""CPU-side checks of the paged attention's boundary: every refusal comes from the host, before anything is launched."""

import ctypes

import pytest
import torch

import paper_2407_21118_amd as P

ONE, ODD = ctypes.c_void_p(256), ctypes.c_void_p(264)       # non-NULL; never dereferenced: the calls are refused first
HUGE = 1 << 40


def desc(**kw):
    a = dict(n_heads=8, d_head=128, group_head_off=[0, 4, 8], k_rank_off=[0, 64, 128], v_rank_off=[0, 64, 128])
    a.update(kw)
    return P.LayerDesc(**a)


GOOD = dict(batch=2, max_len=100, window=10, n_sink=2, q=ONE, q_pos=None, hk=ONE, hv=ONE, n_pages=64, page_rows=16, page_table=ONE,
            table_stride=7, seq_lens=None, Bk=ONE, Bv=ONE, rope=ONE, rope_len=100, out=ONE, workspace=ONE, bytes=HUGE)


def paged(d, **kw):
    a = dict(GOOD, **kw)
    return P.load_library().palu_attn_paged(d.ref() if d else None, a["batch"], a["max_len"], a["window"], a["n_sink"], *rest(a))


def prefix(d, prefix_len=50, **kw):
    a = dict(GOOD, **kw)
    return P.load_library().palu_attn_prefix(d.ref() if d else None, a["batch"], prefix_len, a["max_len"], *rest(a))


def rest(a):
    return [a[k] for k in ("q", "q_pos", "hk", "hv", "n_pages", "page_rows", "page_table", "table_stride", "seq_lens", "Bk", "Bv",
                           "rope", "rope_len", "out", "workspace", "bytes")] + [None]


BAD = [(dict(batch=0), -1), (dict(batch=70000), -2), (dict(max_len=0), -1), (dict(max_len=113, rope_len=113), -1), (dict(rope_len=99), -1),
       (dict(n_pages=0), -1), (dict(page_rows=0), -1), (dict(page_rows=24), -2), (dict(table_stride=0), -1),
       (dict(n_pages=1 << 28), -2), (dict(bytes=8), -3), (dict(page_table=ctypes.c_void_p(258)), -1), (dict(seq_lens=ctypes.c_void_p(258)), -1)]
BAD += [(dict([(name, bad)]), -1) for name in ("q", "hk", "hv", "Bk", "Bv", "rope", "out", "workspace") for bad in (None, ODD)]
BAD += [(dict(page_table=None), -1)]


@pytest.mark.parametrize("call", [paged, prefix])
@pytest.mark.parametrize("kw,status", BAD)
def test_refused_arguments(call, kw, status):
    assert call(desc(), **kw) == status


@pytest.mark.parametrize("call", [paged, prefix])
@pytest.mark.parametrize("kw,status", [
    (dict(k_latent_dtype=P.PALU_I4, k_rank_off=[0, 128, 256]), -2), (dict(v_latent_dtype=P.PALU_I2, v_rank_off=[0, 128, 256]), -2),
    (dict(k_rank_off=[0, 544, 608]), -2), (dict(v_rank_off=[0, 544, 608]), -2), (dict(k_rank_off=[0, 60, 128]), -1), (dict(d_head=64), -2)])
def test_refused_layers(call, kw, status):
    assert call(desc(**kw)) == status
    assert call(None) == -1


def test_refused_windows_and_prefixes():
    assert paged(desc(), window=-1) == -1
    assert paged(desc(), n_sink=-1) == -1
    assert prefix(desc(), -1) == -1
    assert prefix(desc(), 101) == -1


def test_workspace_queries():
    d = desc()
    whole = P.palu_attn_paged_workspace_bytes(d, 4, 16384)
    assert whole > 0 and P.palu_attn_paged_workspace_bytes(d, 4, 16384, 512, 4) <= whole
    assert P.palu_attn_prefix_workspace_bytes(d, 4, 0, 100) > 0 and P.palu_attn_prefix_workspace_bytes(d, 4, 100, 100) > 0
    lib = P.load_library()
    assert lib.palu_attn_paged_workspace_bytes(d.ref(), 4, 100, 0, 0, None) == -1
    assert lib.palu_attn_prefix_workspace_bytes(d.ref(), 4, 10, 100, None) == -1
    out = ctypes.c_size_t(0)
    assert lib.palu_attn_paged_workspace_bytes(d.ref(), 4, 1 << 30, 2 ** 31 - 1, 2 ** 31 - 1, ctypes.byref(out)) == 0
    assert lib.palu_attn_paged_workspace_bytes(d.ref(), 4, 2 ** 31 - 1, 0, 0, ctypes.byref(out)) == -2
    # all layers and sizes stay finite and host-only
    for batch in (1, 7, 65535):
        for n in (1, 63, 64, 65, 1 << 20):
            assert P.palu_attn_prefix_workspace_bytes(d, batch, n // 2, n) > 0


def test_binding_checks_shapes_and_types():
    d = desc()
    with pytest.raises(ValueError):                          # host tensors
        P.palu_attn_paged(d, 1, 16, torch.zeros(1, 8, 128, dtype=torch.float16), None, torch.zeros(1, 16, 128, dtype=torch.float16),
                          torch.zeros(1, 16, 128, dtype=torch.float16), torch.zeros(1, 1, dtype=torch.int32), None,
                          torch.zeros(64 * 512 * 2, dtype=torch.float16), torch.zeros(64 * 512 * 2, dtype=torch.float16),
                          torch.zeros(24576, dtype=torch.uint8), 16)
