"""CPU-side checks of the 4-bit paged cache's boundary: every refusal comes from the host, before anything is launched."""

import ctypes

import pytest

import paper_2407_21118_amd as P

ONE, ODD, TWO = ctypes.c_void_p(256), ctypes.c_void_p(264), ctypes.c_void_p(258)   # non-NULL; never dereferenced: refused first
ODDEST = ctypes.c_void_p(257)
HUGE = 1 << 40


def desc(**kw):
    a = dict(n_heads=8, d_head=128, group_head_off=[0, 4, 8], k_rank_off=[0, 128, 256], v_rank_off=[0, 256, 512],
             k_latent_dtype=P.PALU_I4, v_latent_dtype=P.PALU_I4)
    a.update(kw)
    return P.LayerDesc(**a)


ATTN = dict(batch=2, max_len=100, window=10, n_sink=2, q=ONE, q_pos=None, hk=ONE, hk_scale=ONE, hk_zero=ONE, hv=ONE, hv_scale=ONE, hv_zero=ONE,
            n_pages=64, page_rows=16, page_table=ONE, table_stride=7, seq_lens=None, Bk=ONE, Bv=ONE, rope=ONE, rope_len=100, out=ONE,
            workspace=ONE, bytes=HUGE)


def attend(d, **kw):
    return P.load_library().palu_attn_paged_quant(d.ref() if d else None, *{**ATTN, **kw}.values(), None)


BAD = [(dict(batch=0), -1), (dict(batch=70000), -2), (dict(max_len=0), -1), (dict(max_len=113, rope_len=113), -1), (dict(rope_len=99), -1),
       (dict(n_pages=0), -1), (dict(page_rows=0), -1), (dict(page_rows=24), -2), (dict(table_stride=0), -1), (dict(window=-1), -1),
       (dict(n_sink=-1), -1), (dict(max_len=(1 << 30) + 1, rope_len=1 << 31 - 1, table_stride=1 << 30), -2), (dict(n_pages=1 << 28), -2),
       (dict(bytes=8), -3), (dict(page_table=TWO), -1), (dict(seq_lens=TWO), -1), (dict(q_pos=TWO), -1), (dict(page_table=None), -1)]
BAD += [(dict([(name, bad)]), -1) for name in ("q", "hk", "hv", "Bk", "Bv", "rope", "out", "workspace") for bad in (None, ODD)]
BAD += [(dict([(name, bad)]), -1) for name in ("hk_scale", "hk_zero", "hv_scale", "hv_zero") for bad in (None, ODDEST)]


@pytest.mark.parametrize("kw,status", BAD)
def test_attention_refuses_arguments(kw, status):
    assert attend(desc(), **kw) == status


LAYERS = [(dict(k_latent_dtype=P.PALU_F16), -2), (dict(v_latent_dtype=P.PALU_F16), -2), (dict(k_latent_dtype=P.PALU_I3), -2),
          (dict(v_latent_dtype=P.PALU_I2), -2), (dict(k_rank_off=[0, 640, 768]), -2), (dict(v_rank_off=[0, 640, 768]), -2),
          (dict(k_rank_off=[0, 64, 192]), -1), (dict(quant_block=64), -2), (dict(quant_block=0), -1), (dict(d_head=64), -2),
          (dict(k_latent_dtype=9), -1), (dict(act_dtype=P.PALU_I4), -1)]


@pytest.mark.parametrize("kw,status", LAYERS)
def test_attention_refuses_layers(kw, status):
    out = ctypes.c_size_t(0)
    assert attend(desc(**kw)) == status
    assert P.load_library().palu_attn_paged_quant_workspace_bytes(desc(**kw).ref(), 2, 100, 0, 0, ctypes.byref(out)) == status
    assert attend(None) == -1


def test_large_batches_have_a_launch():
    for heads, max_len in ((8, 1 << 20), (32, 1 << 20), (128, 100)):
        off = [4 * j for j in range(heads // 4 + 1)]
        d = P.LayerDesc(heads, 128, off, [64 * x for x in off], [64 * x for x in off], k_latent_dtype=P.PALU_I4, v_latent_dtype=P.PALU_I4)
        assert P.palu_attn_paged_quant_workspace_bytes(d, 65535, max_len) > 0


def test_attention_workspace():
    lib, out = P.load_library(), ctypes.c_size_t(0)
    for act in (P.PALU_F16, P.PALU_BF16):
        need = P.palu_attn_paged_quant_workspace_bytes(desc(act_dtype=act), 2, 100, 10, 2)
        assert need > 0 and attend(desc(act_dtype=act), bytes=need - 1, page_rows=16) == -3
    assert lib.palu_attn_paged_quant_workspace_bytes(desc().ref(), 2, 100, 0, 0, None) == -1
    assert lib.palu_attn_paged_quant_workspace_bytes(desc().ref(), 0, 100, 0, 0, ctypes.byref(out)) == -1
    # the other entry point goes on refusing quantised pages
    assert lib.palu_attn_paged_workspace_bytes(desc().ref(), 2, 100, 0, 0, ctypes.byref(out)) == -2


ROWS = dict(hk=ONE, hk_stride=256, hv=ONE, hv_stride=512, n_tok=3, k_codes=ONE, k_scale=ONE, k_zero=ONE, v_codes=ONE, v_scale=ONE, v_zero=ONE,
            n_rows=100, row=None)


def write(d, **kw):
    return P.load_library().palu_quant_latent_kv(d.ref() if d else None, *{**ROWS, **kw}.values(), None)


def read(d, **kw):
    a = {**ROWS, **kw}
    order = ("k_codes", "k_scale", "k_zero", "v_codes", "v_scale", "v_zero", "n_rows", "row", "n_tok", "hk", "hk_stride", "hv", "hv_stride")
    return P.load_library().palu_dequant_latent_kv(d.ref() if d else None, *[a[k] for k in order], None)


BAD_ROWS = [(dict(n_tok=-1), -1), (dict(n_rows=0), -1), (dict(n_rows=1 << 31), -1), (dict(row=TWO), -1), (dict(hk_stride=255), -1),
            (dict(hv_stride=0), -1), (dict(hk=ODDEST), -1), (dict(k_codes=TWO), -1), (dict(v_scale=ODDEST), -1), (dict(n_tok=1 << 33), -2),
            (dict(n_tok=1 << 62), -2)]
BAD_ROWS += [(dict([(name, None)]), -1) for name in ("hk", "hv", "k_codes", "k_scale", "k_zero", "v_codes", "v_scale", "v_zero")]


@pytest.mark.parametrize("call", [write, read])
@pytest.mark.parametrize("kw,status", BAD_ROWS)
def test_rows_refuse_arguments(call, kw, status):
    assert call(desc(), **kw) == status


@pytest.mark.parametrize("call", [write, read])
def test_rows_and_layers(call):
    assert call(None) == -1
    assert call(desc(k_latent_dtype=P.PALU_F16, v_latent_dtype=P.PALU_F16)) == -1            # no side to move
    assert call(desc(k_rank_off=[0, 64, 256])) == -1
    assert call(desc(quant_block=64)) == -2
    assert call(desc(), n_tok=0) == 0                                                        # nothing to do, nothing launched
    assert call(desc(), n_tok=0, hk=None, hv=None) == 0
    only_v = desc(k_latent_dtype=P.PALU_F16)                                                 # the other side's arguments are not looked at
    assert call(only_v, n_tok=0, hk=None, hk_stride=0, k_codes=None, k_scale=None, k_zero=None) == 0
    assert call(only_v, v_codes=None) == -1


PROJECT = dict(x=ONE, n_tok=3, Akt=ONE, Ak_scale=ONE, Ak_zero=ONE, Avt=ONE, Av_scale=ONE, Av_zero=ONE, hk=ONE, hk_stride=256, hv=ONE,
               hv_stride=512, dst_row=None)


def project(d, **kw):
    return P.load_library().palu_encode_kv_w4(d.ref() if d else None, *{**PROJECT, **kw}.values(), None)


BAD_PROJECT = [(dict(n_tok=-1), -1), (dict(hk_stride=255), -1), (dict(hv_stride=511), -1), (dict(dst_row=TWO), -1), (dict(hk=ODDEST), -1),
               (dict(Ak_zero=ODDEST), -1)]
BAD_PROJECT += [(dict([(name, bad)]), -1) for name in ("x", "Akt", "Avt") for bad in (None, ODD)]
BAD_PROJECT += [(dict([(name, None)]), -1) for name in ("Ak_scale", "Ak_zero", "Av_scale", "Av_zero", "hk", "hv")]


@pytest.mark.parametrize("kw,status", BAD_PROJECT)
def test_projection_refuses_arguments(kw, status):
    assert project(desc(), **kw) == status


def test_projection_and_layers():
    assert project(None) == -1
    assert project(desc(d_head=64)) == -2
    assert project(desc(), n_tok=0) == 0 and project(desc(), n_tok=0, x=None, hk=None, hv=None) == 0
    assert project(desc(k_latent_dtype=P.PALU_F16, v_latent_dtype=P.PALU_F16, k_rank_off=[0, 60, 256])) == -1
