"""The Python side of the 4-bit paged cache: tensors that do not fit the layer, the batch or each other are refused before the library
sees them.  Host tensors of the right shapes get as far as the last check, which wants them on a device."""

import pytest
import torch

import paper_2407_21118_amd as P

F16, I32, U8 = torch.float16, torch.int32, torch.uint8


def desc(**kw):
    return P.LayerDesc(**{**dict(n_heads=6, d_head=128, group_head_off=[0, 2, 6], k_rank_off=[0, 128, 384], v_rank_off=[0, 256, 384], q_per_kv=3,
                                 k_latent_dtype=P.PALU_I4, v_latent_dtype=P.PALU_I4), **kw})


def zeros(*shape, dtype=F16):
    return torch.zeros(shape, dtype=dtype)


def attention():
    return dict(q=zeros(2, 18, 128), q_pos=zeros(2, dtype=I32), hk=zeros(5, 16, 192, dtype=U8), hk_scale=zeros(5, 16, 3), hk_zero=zeros(5, 16, 3),
                hv=zeros(5, 16, 192, dtype=U8), hv_scale=zeros(5, 16, 3), hv_zero=zeros(5, 16, 3), page_table=zeros(2, 7, dtype=I32),
                seq_lens=zeros(2, dtype=I32), Bk=zeros((128 * 2 + 256 * 4) * 128), Bv=zeros((256 * 2 + 128 * 4) * 128),
                rope_table=zeros(P.palu_rope_table_bytes(128, 100), dtype=U8), rope_table_len=100, out=zeros(2, 18, 128), workspace=zeros(64, dtype=U8))


def rows():
    return dict(hk=zeros(4, 384), hv=zeros(4, 384), k_codes=zeros(9, 192, dtype=U8), k_scale=zeros(9, 3), k_zero=zeros(9, 3),
                v_codes=zeros(9, 192, dtype=U8), v_scale=zeros(9, 3), v_zero=zeros(9, 3))


def weights():
    return dict(x=zeros(4, 2304), Akt=zeros(384, 1152, dtype=U8), Ak_scale=zeros(384, 18), Ak_zero=zeros(384, 18), Avt=zeros(384, 1152, dtype=U8),
                Av_scale=zeros(384, 18), Av_zero=zeros(384, 18), hk=zeros(9, 400), hk_row_stride_elems=400, hv=zeros(9, 384),
                hv_row_stride_elems=384, dst_row=zeros(4, dtype=I32))


CALLS = {"attention": (lambda d=None, **kw: P.palu_attn_paged_quant(d or desc(), 2, 100, **kw), attention),
         "write": (lambda d=None, **kw: P.palu_quant_latent_kv(d or desc(), **kw), lambda: {**rows(), "dst_row": zeros(4, dtype=I32)}),
         "read": (lambda d=None, **kw: P.palu_dequant_latent_kv(d or desc(), **kw), lambda: {**rows(), "src_row": zeros(4, dtype=I32)}),
         "project": (lambda d=None, **kw: P.palu_encode_kv_w4(d or desc(), **kw), weights)}
OPTIONAL = {"attention": ["q_pos", "seq_lens"], "write": ["dst_row"], "read": ["src_row"], "project": ["dst_row"]}


@pytest.mark.parametrize("name", list(CALLS))
def test_what_fits_is_refused_for_its_device_alone(name):
    call, good = CALLS[name]
    with pytest.raises(ValueError, match="device"):
        call(**good())
    with pytest.raises(ValueError, match="device"):
        call(**{**good(), **{k: None for k in OPTIONAL[name]}})


@pytest.mark.parametrize("name,arg", [(n, a) for n in CALLS for a, t in CALLS[n][1]().items()
                                      if isinstance(t, torch.Tensor) and a not in ("rope_table", "workspace")])
def test_types_and_shapes(name, arg):
    call, good = CALLS[name]
    t = good()[arg]
    with pytest.raises(ValueError, match="dtype"):
        call(**{**good(), arg: t.to(torch.float64)})
    if arg in ("hk", "hv") and name == "project":
        with pytest.raises(ValueError, match="hold"):
            call(**{**good(), arg: t[:3], "dst_row": None})
        with pytest.raises(ValueError, match="hold"):
            call(**{**good(), arg + "_row_stride_elems": 383})
        return
    for other in (t[..., :-1], torch.cat([t, t]))[arg == "page_table":]:        # (a narrower page table may hold max_len rows all the same)
        with pytest.raises(ValueError, match="fit|same|shape|dtype|hold|one per"):
            call(**{**good(), arg: other.contiguous()})


def test_layers_of_other_bits():
    for dtype in (P.PALU_I3, P.PALU_I2):
        with pytest.raises(P.PaluError):
            CALLS["attention"][0](desc(k_latent_dtype=dtype), **attention())
    only_v = desc(k_latent_dtype=P.PALU_F16)                       # the key side takes no part: nothing of it is looked at
    for name in ("write", "read"):
        call, good = CALLS[name]
        with pytest.raises(ValueError, match="device"):
            call(only_v, **{**good(), "hk": None, "k_codes": None, "k_scale": None, "k_zero": None})
        with pytest.raises(ValueError, match="dtype"):
            call(only_v, **{**good(), "v_zero": None})


def test_rows_whose_channels_are_apart():
    for name in ("write", "read"):
        call, good = CALLS[name]
        with pytest.raises(ValueError, match="side by side"):
            call(**{**good(), "hk": zeros(384, 4).t()})


@pytest.mark.parametrize("name", ["write", "read"])
@pytest.mark.parametrize("side", ["k", "v"])
def test_nothing_of_a_side_that_is_not_quantised_is_looked_at(name, side):
    call, good = CALLS[name]
    d = desc(**{side + "_latent_dtype": P.PALU_F16})
    for other in (zeros(7, 5), zeros(384, 4).t(), zeros(3, dtype=torch.float64), None):
        codes = None if other is None else zeros(1)
        with pytest.raises(ValueError, match="device"):
            call(d, **{**good(), "h" + side: other, **{side + x: codes for x in ("_codes", "_scale", "_zero")}})


@pytest.mark.parametrize("name", ["write", "read"])
def test_latents_that_are_missing(name):
    call, good = CALLS[name]
    for h in ("hk", "hv"):
        with pytest.raises(ValueError, match="latent rows"):
            call(**{**good(), h: None})
    with pytest.raises(P.PaluError):                           # no side to move
        call(desc(k_latent_dtype=P.PALU_F16, v_latent_dtype=P.PALU_F16), **{k: None for k in good()})
