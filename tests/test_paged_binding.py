"""The Python side of paged attention: tensors that do not fit the layer, the batch or each other are refused before the library sees
them.  Host tensors of the right shapes get as far as the last check, which wants them on a device."""

import pytest
import torch

import paper_2407_21118_amd as P

F16, I32 = torch.float16, torch.int32


def desc(**kw):
    return P.LayerDesc(**{**dict(n_heads=6, d_head=128, group_head_off=[0, 2, 6], k_rank_off=[0, 64, 160], v_rank_off=[0, 32, 96], q_per_kv=3), **kw})


def good():
    return dict(q=torch.zeros(2, 18, 128, dtype=F16), q_pos=torch.zeros(2, dtype=I32), hk=torch.zeros(5, 16, 160, dtype=F16),
                hv=torch.zeros(5, 16, 96, dtype=F16), page_table=torch.zeros(2, 7, dtype=I32), seq_lens=torch.zeros(2, dtype=I32),
                Bk=torch.zeros((64 * 2 + 96 * 4) * 128, dtype=F16), Bv=torch.zeros((32 * 2 + 64 * 4) * 128, dtype=F16),
                rope_table=torch.zeros(P.palu_rope_table_bytes(128, 100), dtype=torch.uint8), rope_table_len=100,
                out=torch.zeros(2, 18, 128, dtype=F16), workspace=torch.zeros(64, dtype=torch.uint8))


FORMS = [lambda **kw: P.palu_attn_paged(desc(), 2, 100, **kw), lambda **kw: P.palu_attn_prefix(desc(), 2, 50, 100, **kw)]


@pytest.mark.parametrize("call", FORMS)
def test_what_fits_is_refused_for_its_device_alone(call):
    with pytest.raises(ValueError, match="device"):
        call(**good())
    with pytest.raises(ValueError, match="device"):
        call(**{**good(), "q_pos": None, "seq_lens": None})


SHAPES = dict(q=[(2, 6, 128), (1, 18, 128)], out=[(2, 6, 128), (3, 18, 128)], q_pos=[(1,), (3,)], seq_lens=[(1,)], page_table=[(1, 7), (3, 7), (14,)],
              hk=[(5, 16, 96), (5, 8, 160), (4, 16, 160), (80, 160), (12800,)], hv=[(5, 16, 160), (5, 8, 96), (80, 96), (7680,)])


@pytest.mark.parametrize("call", FORMS)
@pytest.mark.parametrize("name,shape", [(n, s) for n, shapes in SHAPES.items() for s in shapes])
def test_shapes(call, name, shape):
    with pytest.raises(ValueError, match="fit|same pages"):
        call(**{**good(), name: torch.zeros(shape, dtype=good()[name].dtype)})


@pytest.mark.parametrize("call", FORMS)
@pytest.mark.parametrize("name", ["q", "hk", "hv", "Bk", "Bv", "out", "q_pos", "page_table", "seq_lens"])
def test_types(call, name):
    for dtype in (torch.bfloat16, torch.int64):
        with pytest.raises(ValueError, match="dtype"):
            call(**{**good(), name: good()[name].to(dtype)})


@pytest.mark.parametrize("call", FORMS)
@pytest.mark.parametrize("name", ["Bk", "Bv"])
@pytest.mark.parametrize("off", [-1, -128 * 64, 128])
def test_weights_of_another_size(call, name, off):
    """B_k and B_v hold what the layer's ranks say: one too short would be read behind its end."""
    with pytest.raises(ValueError, match="fit"):
        call(**{**good(), name: torch.zeros(good()[name].numel() + off, dtype=F16)})


@pytest.mark.parametrize("call", FORMS)
def test_angle_tables_too_short(call):
    """rope_table holds rope_table_len positions, whatever its type; a longer one is fine."""
    for n in (1, 32, 96):                                            # (the table goes in steps of 32 positions)
        with pytest.raises(ValueError, match="rope_table"):
            call(**{**good(), "rope_table": torch.zeros(P.palu_rope_table_bytes(128, n), dtype=torch.uint8)})
    with pytest.raises(ValueError, match="rope_table"):
        call(**{**good(), "rope_table": good()["rope_table"][:-1].clone()})
    for table in (good()["rope_table"].view(torch.float32), torch.zeros(P.palu_rope_table_bytes(128, 500), dtype=torch.uint8)):
        with pytest.raises(ValueError, match="device"):
            call(**{**good(), "rope_table": table})


def test_batches_of_more_work_items_than_a_launch_takes():
    """A launch has fewer than 2^32 work items: 128 units of 65535 sequences and blocks of the prefix's rows are more, without these they are not."""
    wide = P.LayerDesc(256, 128, [4 * j for j in range(65)], [512 * j for j in range(65)], [32 * j for j in range(65)])
    with pytest.raises(P.PaluError) as e:
        P.palu_attn_prefix_workspace_bytes(wide, 65535, 32, 64)
    assert e.value.status == -2
    assert P.palu_attn_paged_workspace_bytes(wide, 65535, 32) > 0
