"""Attention over a paged latent cache where its arithmetic can go wrong: what a bfloat16 layer rounds, probabilities far below the
largest, numbers that are none, lengths beyond the bound, page entries out of range."""

import numpy as np
import pytest
import torch

import paper_2407_21118_amd as P
from oracle import palu_oracle as O
from workloads import synth

pytestmark = pytest.mark.gpu

from gpu_util import make_desc, say, torch_dtype  # noqa: E402
from test_gpu_paged import LAYERS, Pool, hold  # noqa: E402


@pytest.mark.parametrize("name,prefix", [("4x256", 0), ("1x64", 0), ("gqa4", 0), ("8x512", 0), ("4x128-384", 0),
                                         ("4x256", 200), ("1x64", 200), ("gqa70", 200), ("3x384-64", 200)])
def test_a_bfloat16_layer_rounds_its_output_alone(name, prefix):
    """The output is the exact one rounded once: off by half a step of its own binade, and by what the sums before it are off.
    Keys and queries are pairs of float16 numbers (2^-21 of a product), composed angles right to 1e-6, so a logit of
    sum(|q k|) / sqrt(128) < 24 is right to 24 * 2.2e-6 = 2^-14.2 and so are probabilities, relative; these and the merged latents
    are pairs of bfloat16 numbers (2^-16 each).  Together 2^-13 of the row's largest output.  A key or a query rounded to
    11 bits moves a logit by up to 2^-11 of the same sum, 2^-9 of the output where few rows carry it."""
    lens = [333, 200, 257] if not prefix else [201 + 7 * i for i in range(21)]
    pool = Pool(LAYERS[name](), "bf16", lens, 16, seed=30, prefix=prefix)
    pool.put(0, 0)
    got = pool.call(pool.device()).double().cpu().numpy()
    ref = pool.reference()
    half = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(ref), 2.0 ** -100))) - 8)
    room = half + 2.0 ** -13 * np.abs(ref).max(-1, keepdims=True)
    off = np.abs(got - ref)
    beyond = np.maximum(off - half, 0) / np.abs(ref).max(-1, keepdims=True)
    say(f"[paged] {name}, prefix {prefix}: beyond half a step by at most {beyond.max():.2e} of the row's largest")
    assert (off <= room).all(), beyond.max()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("q_per_kv", [1, 5])
@pytest.mark.parametrize("at", [0, 2000])
def test_rows_that_one_row_outweighs(at, q_per_kv, dtype):
    """4000 rows of one score under one row whose score is larger by up to 20 (2^-28.9 of its probability) and whose values are zero,
    as a first row may have them: the output is the 4000 rows' alone.  All lie in one split, which shares one running maximum.

    A pair of float16 numbers of probabilities scaled by 2^15 is right to 2^-22 relative or 2^-40 of the largest, whichever is more:
    exp(gap) * 2^-40 of these rows', all of them in the same direction.  Beside it, of the row's largest output: the score's products of
    one sign (gap * 2^-20.5 = 2^-16.2), the float32 sum of 126 tiles (2^-17), and the merged latents, pairs of numbers of which
    the second has steps of 2^-24 (64 of 2^-25 times |B_v| < 0.4 against outputs of 8e-3: 2^-13.4 at their worst, with random signs
    2^-16.4).  Together 2^-14.  bfloat16 pairs keep 2^-16 relative at every size: 2^-14 with the merged latents', too."""
    gaps = [0.0, 5.0, 10.0, 14.0, 16.0, 17.4, 19.0, 20.0]
    layer = synth.uniform_layer(4, 4, 64, rope_theta=0.0, q_per_kv=q_per_kv)     # (no rotation: rows of equal latents score alike)
    desc, n, batch, page = make_desc(layer, dtype), 4001, 256, 64
    assert P.palu_attn_paged_workspace_bytes(desc, batch, n) == P.palu_attn_paged_workspace_bytes(desc, batch, 32)   # one split
    rng = np.random.default_rng(31)
    draw = lambda *s: rng.standard_normal(s)  # noqa: E731
    Bk, Bv = (synth.round_to(draw(64 * 4 * 128) / 8, dtype) for _ in range(2))
    pages = -(-n // page)
    hk, hv = np.full((2, pages * page, 64), np.nan)
    hk[:n], hv[:n] = 0.0, synth.round_to(1000 * (1 + 0.25 * draw(n, 64)), dtype)
    hk[at], hv[at] = synth.round_to(draw(64), dtype), 0.0
    key = (hk[at] @ Bk.reshape(64, 512)).reshape(4, 1, 128)
    key = key * np.sqrt(128) / (key ** 2).sum(-1, keepdims=True)
    q = np.stack([synth.round_to((key * np.array([gaps[(b + i) % 8] for i in range(q_per_kv)])[None, :, None]).reshape(-1, 128), dtype)
                  for b in range(8)])
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(torch_dtype(dtype)).cuda()  # noqa: E731
    got = P.palu_attn_paged(desc, batch, n, dev(q).repeat(batch // 8, 1, 1), None, dev(hk.reshape(pages, page, 64)), dev(hv.reshape(pages, page, 64)),
                            torch.arange(pages, dtype=torch.int32, device="cuda").repeat(batch, 1), None, dev(Bk), dev(Bv),
                            P.palu_rope_table_init(0.0, 128, n), n)
    assert torch.equal(got, got[:8].repeat(batch // 8, 1, 1))
    got = got[:8].double().cpu().numpy()
    both = lambda x: np.repeat(x[None, :n], 8, 0)  # noqa: E731
    ref = O.attn_decode(q, np.full(8, n - 1), both(hk), both(hv), Bk, Bv, layer.group_head_off, layer.k_rank_off, layer.v_rank_off, 128, 0.0,
                        np.arange(n, dtype=np.int32), None, q_per_kv)
    gap = np.array([[gaps[(b + i) % 8] for _ in range(4) for i in range(q_per_kv)] for b in range(8)])
    top = np.abs(ref).max(-1)
    off = np.maximum(np.abs(got - ref) - np.abs(ref) * (2.0 ** -11 if dtype == "f16" else 2.0 ** -8), 0).max(-1) / top
    say(f"[paged] {dtype}, {q_per_kv} queries a head, row {at}: beyond rounding " + " ".join(f"{g}: {off[gap == g].max():.1e}" for g in gaps))
    assert (off <= 2.0 ** -14 + (2.0 ** -40 * np.exp(gap) if dtype == "f16" else 0)).all()


def both_forms(dtype, lens, prefix, seed, layer="4x128", max_len=None):
    pool = Pool(LAYERS[layer](), dtype, lens, 16, seed=seed, prefix=prefix, max_len=max_len)
    pool.put(0, 0)
    return pool, pool.device()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("layer", ["4x128", "gqa4", "8x512"])
@pytest.mark.parametrize("prefix", [0, 300])
def test_a_query_that_is_no_number_answers_none(layer, prefix, dtype):
    """One NaN in the query of one head: that head's output is NaN, every other has the bits that it has without; an idle slot's is zeros."""
    say(f"[nan] {layer} {dtype}, prefix {prefix}")
    pool, d = both_forms(dtype, [700, 0, 333, 450], prefix, 32, layer)
    clean = pool.call(d)
    heads = pool.layer.n_q_heads
    d["q"][0, 2, 5] = d["q"][1] = d["q"][3, heads - 1, 127] = float("nan")
    got = pool.call(d)
    lost = torch.zeros(4, heads, 1, dtype=torch.bool, device="cuda")
    lost[0, 2] = lost[3, heads - 1] = True
    assert torch.equal(got.isnan(), lost.expand_as(got))
    assert torch.equal(got.masked_fill(lost, 0), clean.masked_fill(lost, 0)) and not got[1].any()


@pytest.mark.parametrize("side", ["hk", "hv"])
def test_attended_rows_that_are_no_numbers(side):
    """NaN in five runs of 1 .. 8 tiles of 32 rows in the middle of a sequence, so that some splits hold nothing else whatever their length:
    its outputs are NaN.  Another sequence's have the bits that they have without, and so has its own where a window or its length leaves
    these rows out."""
    pool, d = both_forms("f16", [4032, 3999], 0, 33)
    clean, late, early = pool.call(d), pool.call(d, 500, 4), d["seq_lens"].clone()
    early[0] = 150
    short = pool.call({**d, "seq_lens": early})
    whole = d[side]
    for tiles in (1, 2, 3, 4, 5, 6, 8):
        say(f"[nan] {side}, runs of {tiles} tiles")
        d[side] = whole.clone()
        d[side][d["page_table"][0, 10 * tiles: 20 * tiles].long()] = float("nan")
        got = pool.call(d)
        assert got[0].isnan().all() and torch.equal(got[1], clean[1])
        assert torch.equal(pool.call(d, 500, 4), late)
        if tiles == 1:
            assert torch.equal(pool.call({**d, "seq_lens": early}), short)


@pytest.mark.parametrize("side", ["hk", "hv"])
def test_own_or_shared_rows_that_are_no_numbers(side):
    """NaN in all of one sequence's rows behind the prefix: its outputs alone are NaN.  In the prefix: everyone's, but an idle slot's."""
    pool, d = both_forms("f16", [3900, 3100, 0], 3008, 34)
    clean, whole = pool.call(d), d[side].clone()
    d[side][d["page_table"][0, 188:].long()] = float("nan")
    got = pool.call(d)
    assert got[0].isnan().all() and torch.equal(got[1:], clean[1:])
    for tiles in (1, 2, 3, 4, 5):
        d[side] = whole.clone()
        d[side][d["page_table"][0, 20 * tiles: 30 * tiles].long()] = float("nan")
        got = pool.call(d)
        assert got[:2].isnan().all() and not got[2].any()


def test_values_that_are_no_numbers_under_a_weight_of_zero():
    """A row whose score is 200 above the others', whose splits then weigh exp(-200) = 0 in float32: zero times a NaN among their values
    is NaN, as in the sum that is not split."""
    pool = Pool(LAYERS["norope"](), "f16", [4032], 16, seed=35)
    pool.rows[0][1:, : pool.layer.R_k] = 0.0
    key = np.concatenate([(pool.rows[0][0, 128 * j: 128 * j + 128] @ pool.Bk[j * 65536:(j + 1) * 65536].reshape(128, 512)).reshape(4, 128) for j in (0, 1)])
    pool.q = synth.round_to(200 * np.sqrt(128) * key / (key ** 2).sum(-1, keepdims=True), "f16")[None]
    pool.put(0, 0)
    d = pool.device()
    hold(pool.call(d), pool.reference(), "f16")
    d["hv"][d["page_table"][0, 100: 180].long(), 3, 130] = float("nan")
    got = pool.call(d)
    assert torch.isfinite(got[0, :4]).all() and got[0, 4:].isnan().all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_a_query_beyond_the_range_does_not_answer_zeros(dtype):
    """A rotated query above 65504 / (8 log2(e) / sqrt(128)) = 6.4e4 has no float16 pair: its head's output is NaN, not an idle slot's."""
    pool, d = both_forms(dtype, [100, 200], 0, 34)
    clean = pool.call(d)
    d["q"][0, 1] = 6.0e4                                             # (turned by some angle, a pair of 6e4 has an entry of more than 6.4e4)
    got = pool.call(d)
    assert got[0, 1].isnan().all()
    got[0, 1] = clean[0, 1]
    assert torch.equal(got, clean)


@pytest.mark.parametrize("prefix", [0, 100])
def test_lengths_beyond_their_bound(prefix):
    """seq_lens above max_len count as max_len, for the rows and for the query's position, also where the angle table goes on; below 0 as 0."""
    pool, d = both_forms("f16", [260, 260, 200], prefix, 36)
    d["rope_table"], d["rope_table_len"] = P.palu_rope_table_init(pool.layer.rope_theta, 128, 1000), 1000
    right = pool.call(d)
    d["seq_lens"][:2] = torch.tensor([267, 2 ** 31 - 1])
    assert torch.equal(pool.call(d), right)
    hold(right, pool.reference(), "f16")
    d["seq_lens"][1] = -5
    got = pool.call(d)
    assert torch.equal(got[[0, 2]], right[[0, 2]]) and not got[1].any()


def test_device_tensors_that_do_not_fit_are_refused():
    """Before anything is launched: strides, types, shapes, sizes."""
    for prefix in (0, 32):
        pool, d = both_forms("f16", [100, 60], prefix, 37)
        bad = {name: torch.zeros(*d[name].shape[:-1], 2 * d[name].shape[-1], dtype=d[name].dtype, device="cuda")[..., ::2]
               for name in ("q", "hk", "hv", "page_table", "Bk", "Bv", "seq_lens")}
        bad["rope_table"] = d["rope_table"][:-16].clone()
        for name, x in bad.items():
            with pytest.raises(ValueError):
                pool.call({**d, name: x})
        for name in ("q", "hk", "Bv", "page_table", "seq_lens"):
            for x in (d[name].float(), d[name][:1].clone()):
                with pytest.raises(ValueError):
                    pool.call({**d, name: x})
        for kw in (dict(out=d["q"][:1].clone()), dict(out=torch.empty(2, 8, 256, dtype=torch.float16, device="cuda")[..., ::2])):
            with pytest.raises(ValueError):
                pool.call(d, **kw)
        with pytest.raises(P.PaluError):
            pool.call(d, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
        hold(pool.call(d), pool.reference(), "f16")


@pytest.mark.parametrize("entry,page", [(60, 59), (2 ** 31 - 1, 59), (-1, 0), (-2 ** 31, 0)])
def test_page_entries_out_of_range_are_the_nearest_page(entry, page):
    """Against the oracle over the rows of the first or the last page, which hold numbers of their own."""
    pool = Pool(LAYERS["4x128"](), "f16", [300, 40, 0], 16, seed=38)
    rng = np.random.default_rng(39)
    pool.table = 1 + rng.permutation(58)[:57].reshape(3, 19).astype(np.int32)    # (not the first of the 60 pages, nor the last)
    pool.put(0, 0)
    for x in (pool.hk, pool.hv):
        for p in (0, 59):
            x[p] = synth.round_to(rng.standard_normal(x[p].shape), "f16")
    pool.table[1, 1] = entry
    d = pool.device()
    got = pool.call(d)
    pool.rows[1][16:32] = np.concatenate([pool.hk[page], pool.hv[page]], -1)
    hold(got, pool.reference(), "f16")


@pytest.mark.parametrize("batch", [3, 40])
def test_the_first_slot_of_a_batch_idle_behind_its_prefix(batch):
    """Sequence 0 has ended: its page table goes on naming the shared pages, its output is zeros, and the others' are as with it."""
    pool, d = both_forms("f16", [290 + (7 * i) % 90 for i in range(batch)], 275, 40)
    whole = pool.call(d)
    d["seq_lens"][0] = 0
    got = pool.call(d)
    assert not got[0].any() and torch.equal(got[1:], whole[1:])
    hold(whole, pool.reference(), "f16")


def test_queries_of_one_sequence_behind_a_prefix():
    """A speculative-decoding check: three entries each of two sequences, with one page-table row and lengths of their own."""
    pool = Pool(LAYERS["4x128"](), "f16", [400, 400, 400, 330, 330, 330], 16, seed=41, prefix=300)
    pool.put(0, 0)
    d = pool.device()
    d["page_table"][1:3], d["page_table"][4:] = d["page_table"][0], d["page_table"][3]
    pool.rows[1] = pool.rows[2] = pool.rows[0]
    pool.rows[4] = pool.rows[5] = pool.rows[3]
    pool.lens = [400, 399, 398, 330, 329, 301]
    d["seq_lens"] = torch.tensor(pool.lens, dtype=torch.int32, device="cuda")
    hold(pool.call(d), pool.reference(), "f16")
